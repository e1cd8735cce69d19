// Causal attention of new tokens over the paged cache, for gfx950.
//
//   out[i, h] = sum_t softmax_t(scale * q[i, h] . K[t, h / G]) * V[t, h / G]     for t <= p_i, the position of token i
//
// A workgroup has the rows (token, head of the group) of some tokens of one request and KV head, 32 to a wavefront, and goes over the keys that
// the last of them sees, 64 at a time.  K and V of those are staged in LDS as bf16 once for all rows.  Per 32 keys, lane = 32*h + n:
//   S^T = K . Q^T   D/16 v_mfma_f32_32x32x16_bf16.  A = K rows, lane (n, h) has the 16 bytes at dims 16*jj + 8*h of key n; B = q, which stays in
//         registers, lane (n, h) has the same dims of row n.  The result leaves lane (n, h) with row n's scores of keys 8*(r / 4) + 4*h + r % 4.
//   P     = exp2(score - m), rounded to bf16.  A lane has scores of one row alone, so that maximum, sum and rescale stay in the lane but for one
//         exchange between the halves when the maximum is raised.
//   O^T  += V^T . P^T  D/32 times two for 32 keys.  P is the B operand as it came out; A takes dims in rows out of V's rows of dims by
//         transposing reads of LDS, four keys of 16 dims to 16 lanes, in the order of keys that P has.
// The running maximum is only raised when a score exceeds it by more than 2^8, as in the decode kernels.
#include "attn_partial.h"
#include "pkv_kernels.h"

#include <type_traits>

namespace pkv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef const int32_t __attribute__((address_space(4))) * ScalarLoad;

constexpr float kLazyLog2 = 8.f;
constexpr int kRawBuffer = 0x00020000;
constexpr int kUnits = kKeyTile / kBlockTokens;   // of a tile
constexpr int kWindowTiles = 64 / kUnits;         // whose units a wavefront's lanes describe

__host__ __device__ constexpr int prompt_waves(int D) { return D == 256 ? 4 : 8; }

// A workgroup's tokens: `first` to `first + count` of the call, of request s, at position `at` and on.
struct Tokens {
  int s, first, count, at;
};
// Slots of `per` tokens: request s has slots start / per + s and on, one or none of them empty.
__device__ __forceinline__ Tokens tokens_of(const PromptLaunch& a, int slot, int per) {
  int s, from, end;
  if (!a.token_starts) {
    s = from = slot;
    end = from + 1;
    if (s >= a.S) return {0, 0, 0, 0};
    slot = 0;
  } else {
    // the last request whose slots begin at or before this one: one look of 64 lanes up to 63 requests, else two, kMaxSeqs being 32 times 64
    const int lane = threadIdx.x & 63, step = (a.S >> 6) + 1;
    auto start = [&](int i) { return min(max(a.token_starts[min(i, a.S)], 0), a.T); };
    int base = 0;
    if (step > 1) {
      const int i = lane * step;
      base = max(__popcll(__ballot(i < a.S && start(i) / per + i <= slot)) - 1, 0) * step;
    }
    const int j = base + lane, at = start(j);
    const int found = __popcll(__ballot(j < a.S && lane < 63 && at / per + j <= slot)) - 1;
    if (found < 0) return {0, 0, 0, 0};
    s = base + found;
    from = __builtin_amdgcn_readlane(at, found);
    end = __builtin_amdgcn_readlane(at, found + 1);
    slot -= from / per + s;
  }
  const int L = min(max(*(ScalarLoad)(a.context_lens + s), 0), a.max_ctx);
  const int n = end - from;
  // tokens before position 0 have none
  const int skip = max(n - L, 0);
  const int lo = max(slot * per, skip), hi = min((slot + 1) * per, n);
  return {s, from + lo, max(hi - lo, 0), L - n + lo};
}

__device__ __forceinline__ u32x2 widen(uint32_t w, float scale) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, true))};
}

// Places in LDS, in bytes: 16-byte piece p of key t.  K is read 16 bytes a lane, a key to a lane; V 8 bytes a lane, four keys of 64 bytes to half
// a wavefront.  No conflicts in either, nor where they are written.
template <int kD> __device__ __forceinline__ int k_place(int t, int p) {
  constexpr int kPieces = kD / 8;
  const int turn = kPieces == 8 ? (t >> 1) & 7 : t & 15;
  return (t * kPieces + (p ^ turn)) * 16;
}
template <int kD> __device__ __forceinline__ int v_place(int t, int p) {
  constexpr int kPieces = kD / 8;
  const int turn = kPieces == 8 ? (t >> 1) & 1 : t & 3;
  return (t * kPieces + (p ^ (turn << 2))) * 16;
}

template <int kD, int kFormat>
__global__ __launch_bounds__(prompt_waves(kD) * 64, kD == 256 ? 1 : 2) void prompt_attn_kernel(PromptLaunch a, int per, int slots, uint32_t group_inverse) {
  constexpr int kWaves = prompt_waves(kD), kThreads = kWaves * 64, kSteps = kD / 16, kTiles = kD / 32;
  constexpr int kTileBytes = kKeyTile * kD * 2;
  constexpr int kElem = kFormat == 0 ? 2 : 1;
  constexpr int kSource = kKeyTile * kD * kElem / 16;            // 16-byte pieces of a tile as the pool has it
  constexpr int kLoads = (kSource + kThreads - 1) / kThreads;    // of a lane
  constexpr int kPerToken = kD * kElem / 16;
  __shared__ __align__(16) char lds[4 * kTileBytes];             // K and V of two tiles in turn
  __shared__ int not_finite[2];                                  // the last tile of whose V something is not finite, plus 1

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int kvh = blockIdx.x % a.Hkv;
  const int slot = slots - 1 - (int)(blockIdx.x / a.Hkv);        // late tokens see most: they begin first
  const Tokens tok = tokens_of(a, slot, per);
  const int keys = tok.at + tok.count;                           // that the last one sees
  const int tiles = (keys + kKeyTile - 1) / kKeyTile;
  const int from = blockIdx.y * a.piece, to = min(from + a.piece, tiles);
  if (tok.count <= 0 || from >= to) return;

  // This lane's row, and the last key that it sees; rows behind the last are computed along with it.
  const int row = 32 * wave + n;
  int which = (int)((row * group_inverse) >> 16);                // row / G
  const int head = row - which * a.G;
  const bool live = which < tok.count;
  which = min(which, tok.count - 1);
  const int64_t q_row = ((int64_t)(tok.first + which) * a.Hq + kvh * a.G + head) * kD;
  const int last_key = tok.at + which;
  const int wave_from = __builtin_amdgcn_readlane(last_key, 0), wave_to = __builtin_amdgcn_readlane(last_key, 31);
  const bool idle = __builtin_amdgcn_readfirstlane(!__any(live));

  bf16x8 q[kSteps];
  const bool negative = a.scale_log2e < 0.f;
  const float scale = __builtin_fabsf(a.scale_log2e);
#pragma unroll
  for (int jj = 0; jj < kSteps; ++jj) {
    u32x4 x = *(const u32x4*)(a.q + q_row + 16 * jj + 8 * h);
    if (negative) x ^= 0x80008000u;
    q[jj] = __builtin_bit_cast(bf16x8, x);
  }

  // Units of the context: one to a lane, a window of 64 at a time and the next one ahead.
  struct Window {
    int slab;       // 16 keys of the KV head, counted from the pool's start; -1: not to be read
    int scales;     // kBlkPools: of K, of V
  };
  const int log_units = a.log_block - 4;
  const int context = tok.at + tok.count;   // keys behind this are not seen
  int refused = 0;
  auto describe = [&](int tile) -> Window {
    const int u = kUnits * tile + lane;
    Window w = {-1, 0};
    const bool here = u >= kUnits * from && u * kBlockTokens < context && u < kUnits * to;
    int id = -1;
    if (here) id = a.block_tables[(int64_t)tok.s * a.MAXB + (u >> log_units)];
    const bool mapped = (unsigned)id < (unsigned)a.NB;           // ids outside the pool are never followed
    refused += __popcll(__ballot(here && !mapped));
    if (mapped) {
      w.slab = ((id * a.Hkv + kvh) << log_units) + (u & ((1 << log_units) - 1));
      if constexpr (kFormat == kBlkPools) {
        const int64_t at = (int64_t)id * scale_row_bytes(a.Hkv) + kvh;
        w.scales = a.k_scales[at] | a.v_scales[at] << 8;
      }
    }
    return w;
  };
  int window_at = from / kWindowTiles * kWindowTiles;
  Window now = describe(window_at), then = describe(window_at + kWindowTiles);

  // A tile on its way: out of memory into registers, from there into LDS.
  u32x4 kr[kLoads], vr[kLoads];
  float ks[kLoads], vs[kLoads];
  uint32_t unmapped = 0;      // of the tile that was asked for last: a bit for each key's unit that is not there
  auto ask = [&](int tile) {
    if (tile >= window_at + kWindowTiles) {
      now = then;
      window_at += kWindowTiles;
      then = describe(window_at + kWindowTiles);
    }
    const int u0 = kUnits * (tile - window_at);
    unmapped = 0;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) unmapped |= (__builtin_amdgcn_readlane(now.slab, u0 + u) < 0) << u;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = i * kThreads + wave * 64;                // the wavefront's first
      const int u = piece / kPerToken / kBlockTokens;
      if (kSource % kThreads != 0 && piece >= kSource) break;
      const int slab = __builtin_amdgcn_readlane(now.slab, u0 + u);
      const int rows = min(kBlockTokens, context - kKeyTile * tile - kBlockTokens * u);
      const int64_t at = (int64_t)max(slab, 0) * (kBlockTokens * kD * kElem);
      const int bytes = slab < 0 || rows <= 0 ? 0 : rows * kD * kElem;
      const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.k_pool + at), 0, bytes, kRawBuffer);
      const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.v_pool + at), 0, bytes, kRawBuffer);
      const int offset = 16 * ((piece + lane) % (kPerToken * kBlockTokens));
      kr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kb, offset, 0, 0));
      vr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vb, offset, 0, 0));
      if constexpr (kFormat == kBlkPools) {
        const int both = __builtin_amdgcn_readlane(now.scales, u0 + u);
        ks[i] = __uint_as_float((uint32_t)(both & 0xff) << 23);
        vs[i] = __uint_as_float((uint32_t)(both >> 8) << 23);
      } else {
        ks[i] = vs[i] = 1.f;
      }
    }
  };
  auto put = [&](int tile, char* k_lds, char* v_lds, int* flag, bool look) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = i * kThreads + threadIdx.x;
      if (kSource % kThreads != 0 && piece >= kSource) break;
      const int t = piece / kPerToken, p = piece % kPerToken;
      if constexpr (kFormat == 0) {
        *(u32x4*)(k_lds + k_place<kD>(t, p)) = kr[i];
        *(u32x4*)(v_lds + v_place<kD>(t, p)) = vr[i];
      } else {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const u32x2 k0 = widen(kr[i][2 * z], ks[i]), k1 = widen(kr[i][2 * z + 1], ks[i]);
          *(u32x4*)(k_lds + k_place<kD>(t, 2 * p + z)) = u32x4{k0.x, k0.y, k1.x, k1.y};
          const u32x2 v0 = widen(vr[i][2 * z], vs[i]), v1 = widen(vr[i][2 * z + 1], vs[i]);
          *(u32x4*)(v_lds + v_place<kD>(t, 2 * p + z)) = u32x4{v0.x, v0.y, v1.x, v1.y};
        }
      }
      if (look) {   // a weight of zero does not silence what is not finite
        bool bad = false;
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const uint32_t w = vr[i][z];
          if constexpr (kFormat == 0) bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
          else bad |= (w & 0x7fu) == 0x7fu || (w & 0x7f00u) == 0x7f00u || (w & 0x7f0000u) == 0x7f0000u || (w & 0x7f000000u) == 0x7f000000u;
        }
        if constexpr (kFormat == kBlkPools) bad |= !(vs[i] < 0x1p120f);
        if (bad) *flag = tile + 1;
      }
    }
  };

  float m = kNegInf, l = 0.f;   // of row n: the reference maximum in log2 units, this lane's part of the sum
  f32x16 o[kTiles];             // o[d][r]: row n, dim 32*d + 8*(r / 4) + 4*h + r % 4
#pragma unroll
  for (int d = 0; d < kTiles; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;

  // V's operand of keys 16*step .. +15, dims 32*d .. +31
  const int v_key = 4 * h + ((lane & 15) >> 2), v_dim = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);   // this lane's part of what 16 lanes transpose
  auto v_operand = [&](const char* v_lds, int step, int d) -> u32x4 {
    typedef __attribute__((address_space(3))) s16x4* Place;
    const int p = (32 * d + v_dim) >> 3, byte = 2 * (v_dim & 7);
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(v_lds + v_place<kD>(16 * step + v_key, p) + byte));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(v_lds + v_place<kD>(16 * step + 8 + v_key, p) + byte));
    const u32x2 xx = __builtin_bit_cast(u32x2, x), yy = __builtin_bit_cast(u32x2, y);
    return u32x4{xx.x, xx.y, yy.x, yy.y};
  };

  auto attend = [&](const char* k_lds, const char* v_lds, int tile, uint32_t gone, bool some_not_finite) __attribute__((always_inline)) {
    f32x16 s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
      for (int jj = 0; jj < kSteps; ++jj) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, *(const u32x4*)(k_lds + k_place<kD>(32 * b + n, 2 * jj + h)));
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[jj], s[b], 0, 0, 0);
      }
    }
    const int key0 = kKeyTile * tile;
    const bool edge = gone != 0 || key0 + kKeyTile - 1 > wave_from;
    uint32_t seen[2];   // bit r: does the row see that key
    if (edge) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        seen[b] = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * b + 8 * (r >> 2) + 4 * h + (r & 3);
          const bool ok = key0 + key <= last_key && !((gone >> (2 * b + (r >> 3))) & 1);
          seen[b] |= (uint32_t)ok << r;
          s[b][r] = ok ? s[b][r] : kNegInf;
        }
      }
    }
    float most = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) most = fmaxf(fmaxf(most, s[0][r]), s[1][r]);
    if (__any(most * scale > m + kLazyLog2)) {
      most = fmaxf(most, __shfl_xor(most, 32)) * scale;
      const float raised = fmaxf(m, most);
      const float alpha = raised == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m - raised);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m = raised;
    }
    u32x4 p[4];   // weights of keys 16*step .. +15, the B operand
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], scale, -m));
        if (edge) w = (seen[b] >> r) & 1 ? w : 0.f;   // m may still be -inf here
        s[b][r] = w;
        sum[b] += w;
      }
#pragma unroll
      for (int z = 0; z < 8; ++z) p[2 * b + (z >> 2)][z & 3] = pack_bf16(s[b][2 * z], s[b][2 * z + 1]);
    }
    l += sum[0] + sum[1];
    if (__builtin_expect(edge && some_not_finite, 0)) {
      // What is not finite in V reaches the rows that see its key and no other.  All else first, then key by key.
#pragma unroll
      for (int step = 0; step < 4; ++step) {
#pragma unroll 1
        for (int key = -1; key < 16; ++key) {
          const bool mine = key < 0 || h == ((key >> 2) & 1);
          const int element = (key & 3) + 4 * (key >> 3);
          const bool sees = key0 + 16 * step + key <= last_key;
#pragma unroll
          for (int d = 0; d < kTiles; ++d) {
            u32x4 v = v_operand(v_lds, step, d);
#pragma unroll
            for (int z = 0; z < 8; ++z) {
              const uint32_t half = z & 1 ? 0xffff0000u : 0xffffu;
              const bool finite = (v[z >> 1] & half & 0x7f807f80u) != (half & 0x7f807f80u);
              const bool keep = key < 0 ? finite : mine && z == element && !finite;
              v[z >> 1] &= keep ? 0xffffffffu : ~half;
            }
            const f32x16 zero = {};
            const f32x16 add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p[step]), zero, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = key < 0 || sees ? o[d][r] + add[r] : o[d][r];
          }
        }
      }
      return;
    }
#pragma unroll
    for (int step = 0; step < 4; ++step)
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_operand(v_lds, step, d)), __builtin_bit_cast(bf16x8, p[step]), o[d],
                                                       0, 0, 0);
  };

  if (threadIdx.x < 2) not_finite[threadIdx.x] = 0;
  __syncthreads();
  ask(from);
  for (int tile = from; tile < to; ++tile) {
    const int turn = (tile - from) & 1;
    char *k_lds = lds + 2 * turn * kTileBytes, *v_lds = k_lds + kTileBytes;
    const uint32_t gone = unmapped;
    put(tile, k_lds, v_lds, not_finite + turn, kKeyTile * tile + kKeyTile - 1 > tok.at);
    if (tile + 1 < to) ask(tile + 1);
    __syncthreads();
    if (!idle && kKeyTile * tile <= wave_to) attend(k_lds, v_lds, tile, gone, not_finite[turn] == tile + 1);
  }
  if (a.id_faults && refused && threadIdx.x == 0) atomicAdd(a.id_faults, refused);

  if (!live) return;
  const float total = l + __shfl_xor(l, 32);
  if (tiles <= a.piece) {
    const float inv = inverse(total, a.out_scale);
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(u32x2*)(a.out + q_row + 32 * d + 8 * g + 4 * h) =
            finish_row4(f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]}, inv);
  } else {
    float* part = a.parts + (int64_t)blockIdx.y * a.T * a.Hq * kD + q_row;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(part + 32 * d + 8 * g + 4 * h) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    if (h == 0) *(f32x2*)(a.stats + ((int64_t)blockIdx.y * a.T * a.Hq + q_row / kD) * 2) = f32x2{m, total};
  }
}

// The rows of contexts that were cut, from their pieces: D / 4 lanes to a row.
template <int kD>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptLaunch a, int per) {
  constexpr int kLanes = kD / 4, kAtOnce = 4;
  const int token = blockIdx.x;
  // the slot of a token is found the way its workgroup was: all of its request's slots begin at or before it
  int s = token, from = token, end = token + 1;
  if (a.token_starts) {
    s = -1;
    for (int step = 1 << (31 - __clz(a.S)); step > 0; step >>= 1)
      if (s + step < a.S && a.token_starts[s + step] <= token) s += step;
    if (s < 0) return;
    from = min(max(a.token_starts[s], 0), a.T);
    end = min(max(a.token_starts[s + 1], 0), a.T);
  }
  if (token < from || token >= end) return;
  const int L = min(max(a.context_lens[s], 0), a.max_ctx), n = end - from;
  if (token - from < n - L) return;
  const int last = min(((token - from) / per + 1) * per, n) - 1;     // of its workgroup's tokens
  const int tiles = (L - n + last + 1 + kKeyTile - 1) / kKeyTile;
  if (tiles <= a.piece) return;
  const int count = (tiles + a.piece - 1) / a.piece;
  const int64_t rows = (int64_t)a.T * a.Hq;
  for (int head = blockIdx.y * (256 / kLanes) + threadIdx.x / kLanes; head < a.Hq; head += gridDim.y * (256 / kLanes)) {
    const int64_t row = (int64_t)token * a.Hq + head;
    const int dim = 4 * (threadIdx.x % kLanes);
    Partial p = kNothing;
    for (int i = 0; i < count; i += kAtOnce) {
      f32x2 ml[kAtOnce];
      f32x4 x[kAtOnce];
#pragma unroll
      for (int z = 0; z < kAtOnce; ++z) {
        const int64_t at = min(i + z, count - 1) * rows + row;
        ml[z] = *(const f32x2*)(a.stats + 2 * at);
        x[z] = *(const f32x4*)(a.parts + at * kD + dim);
      }
#pragma unroll
      for (int z = 0; z < kAtOnce; ++z)
        if (i + z >= count) ml[z] = f32x2{kNegInf, 0.f};
      fold(p, ml, x);
    }
    *(u32x2*)(a.out + row * kD + dim) = finish_row4(p.x, inverse(p.l, a.out_scale));
  }
}

template <int kD, int kFormat>
void launch(const PromptLaunch& a, const PromptPlan& plan, hipStream_t stream) {
  const dim3 grid((unsigned)(plan.slots * a.Hkv), plan.pieces), block(prompt_waves(kD) * 64);
  hipLaunchKernelGGL((prompt_attn_kernel<kD, kFormat>), grid, block, 0, stream, a, plan.tokens, (int)plan.slots, 65536u / a.G + 1);
  if (plan.pieces > 1) {
    const int heads = 256 / (kD / 4);
    hipLaunchKernelGGL((prompt_join_kernel<kD>), dim3(a.T, (a.Hq + heads - 1) / heads), dim3(256), 0, stream, a, plan.tokens);
  }
}
template <int kD>
void launch_format(const PromptLaunch& a, const PromptPlan& plan, hipStream_t stream) {
  if (a.kv_fp8 == kBlkPools) launch<kD, kBlkPools>(a, plan, stream);
  else if (a.kv_fp8) launch<kD, 1>(a, plan, stream);
  else launch<kD, 0>(a, plan, stream);
}

}  // namespace

PromptPlan prompt_plan(int64_t T, int S, int Hkv, int G, int D, int max_ctx) {
  PromptPlan p;
  p.rows = 32 * prompt_waves(D);
  p.tokens = p.rows / G;
  p.slots = T / p.tokens + S;
  const int64_t tiles = ((int64_t)max_ctx + kKeyTile - 1) / kKeyTile, groups = p.slots * Hkv;
  const int64_t least = 8;
  int64_t piece = groups * tiles / 1024;
  if (piece < least) piece = least;
  if (piece > tiles) piece = tiles > 0 ? tiles : 1;
  p.piece = (int)piece;
  p.pieces = (int)(tiles > 0 ? (tiles + piece - 1) / piece : 1);
  return p;
}

hipError_t launch_prompt(const PromptLaunch& a, const PromptPlan& plan, hipStream_t stream) {
  if (a.D == 64) launch_format<64>(a, plan, stream);
  else if (a.D == 128) launch_format<128>(a, plan, stream);
  else if (a.D == 256) launch_format<256>(a, plan, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
