// New tokens on their way into the cache, for gfx950: queries and keys normalised head by head and rotated to their positions, queries to
// the attention's input, keys and values to their slots of the paged pools, in one pass over the rows that a fused projection gives.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          a row of D values, where there are weights
//   (a, b) -> (a cos - b sin, b cos + a sin)    pairs (j, j + R/2) or (2j, 2j + 1) of the first R dims; cos and sin from the position's row
//
// in fp32, rounded once to what is stored.  Prompts are bound by memory, each row in and out once (16 of 100..2000 tokens on 40/8 heads, 505 MB,
// 94 us: 5.4 TB/s, a 1 GiB copy 4.8), a step's few tokens by the launch and three round trips: lengths, the position's row and table entry,
// stores.  D / 8 lanes have a row, and a lane two pieces of four dims: with pairs (j, j + R/2) those of both
// halves, so that a rotation stays in the lane, else (and behind the first R dims) eight in a row.  The sum of squares is all that lanes
// exchange.
#include "fp4.h"
#include "pkv_kernels.h"

namespace pkv {
namespace {

constexpr int kThreads = 256;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
// Two pieces of four dims.
struct Raw {
  u32x2 piece[2];
};
__device__ __forceinline__ void unpack(const Raw& w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w.piece[i >> 1][i & 1] << 16);
    x[2 * i + 1] = __uint_as_float(w.piece[i >> 1][i & 1] & 0xffff0000u);
  }
}
__device__ __forceinline__ Raw load(const uint16_t* row, int p0, int p1) { return Raw{{*(const u32x2*)(row + p0), *(const u32x2*)(row + p1)}}; }
__device__ __forceinline__ float to_range(float y) {
  return (y != y) ? y : fminf(fmaxf(y, -448.f), 448.f);   // NaN stays NaN
}

// A lane's pieces, which begin at dims p0 and p1, into a row; nontemporal, as nothing of a prompt is read again soon: 16 prompts of 100..2000 tokens on
// 40/8 heads 105 us with ordinary stores, 100 this way, 24 pieces of 1..900 in e4m3 at D = 64 29.5 and 24.2; nontemporal loads gain nothing and cost
// 4 us where the projection's rows are still on chip.
__device__ __forceinline__ void put_bf16(char* row, int p0, int p1, const float (&y)[8]) {
  __builtin_nontemporal_store(u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])}, (u32x2*)(row + 2 * p0));
  __builtin_nontemporal_store(u32x2{pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])}, (u32x2*)(row + 2 * p1));
}
// Divided by the pool's scale, clamped to the format's range and rounded to nearest even by the hardware conversion.  `inverse`: the scale's
// rounded reciprocal, or 0.  With it a product and its remainder give the rounded quotient (Markstein's theorem) in three operations instead
// of ten, wherever the quotient is in range.
__device__ __forceinline__ void put_fp8(char* row, int p0, int p1, const float (&y)[8], float scale, float inverse) {
  float z[8];
  if (inverse != 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = y[i] * inverse, exact = __builtin_fmaf(__builtin_fmaf(-q, scale, y[i]), inverse, q);
      z[i] = to_range(__builtin_fabsf(q) < 512.f ? exact : q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = to_range(y[i] / scale);
  }
  int b[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    b[i] = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i + 2], z[4 * i + 3], __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i], z[4 * i + 1], 0, false), true);
  __builtin_nontemporal_store(b[0], (int*)(row + p0));
  __builtin_nontemporal_store(b[1], (int*)(row + p1));
}
// Eight dims in a row of token t of a tile, `chunk` of their KV head's row.  The scale of a group of 32 dims, which are four lanes', is the
// smallest power of two with which none is rounded past 6: 4 to 7 of it are in the largest.  Between 2^-120 and 2^125, so that no product with
// a code leaves the range of normal numbers.  The hardware's conversion rounds to nearest even and holds what is larger at 6; NaN is in the
// scale.
template <int kD>
__device__ __forceinline__ void put_fp4(char* tile, int t, int chunk, const float (&y)[8], bool is_v) {
  uint32_t most = 0;   // of the magnitudes' bits: NaN is above infinity
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(y[i]) & 0x7fffffffu);
  most = max(most, (uint32_t)__shfl_xor((int)most, 1));
  most = max(most, (uint32_t)__shfl_xor((int)most, 2));
  const int e = (int)(most >> 23) - 2 + ((most & 0x7fffff) >= 0x600000);
  const uint32_t byte = min(max(e, 7), 252);
  const float scale = __uint_as_float(byte << 23);
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  if (!is_v) {
    *(uint32_t*)(tile + fp4_k_place(chunk, t)) = w;
  } else if constexpr (kD == 64) {
    *(uint16_t*)(tile + fp4_v_place(kD, 8 * chunk, t)) = (uint16_t)w;
    *(uint16_t*)(tile + fp4_v_place(kD, 8 * chunk + 4, t)) = (uint16_t)(w >> 16);
  } else {
    *(uint32_t*)(tile + fp4_v_place(kD, 8 * chunk, t)) = w;
  }
  if ((chunk & 3) == 0) *(uint8_t*)(tile + fp4_scale_place(kD, chunk >> 2, t)) = most > 0x7f800000u ? 255 : byte;
}

// A token's request and position (< 0: it has none).
struct TokenAt {
  int request, position;
};
__device__ __forceinline__ TokenAt token_at(const RopeLaunch& a, int token) {
  typedef const int32_t __attribute__((address_space(4))) * ScalarLoad;
  int s = token, len;
  uint32_t behind = 1;   // tokens of the request from this one on
  if (a.token_starts) {
    // The last request that begins at or before the token: one look of 64 lanes up to 63 requests, else two, kMaxSeqs being 32 times 64.  Its
    // length and where the next one begins come with the last look.
    const int lane = threadIdx.x & 63, step = (a.S >> 6) + 1;
    int base = 0;
    if (step > 1) {
      const int i = lane * step;
      const int begin = i < a.S ? a.token_starts[i] : INT32_MAX;
      base = max(__popcll(__ballot(begin <= token)) - 1, 0) * step;
    }
    const int j = base + lane;
    const int at = j <= a.S ? a.token_starts[j] : INT32_MAX, length = j < a.S ? a.context_lens[j] : 0;
    const int found = __popcll(__ballot(j < a.S && lane < 63 && at <= token)) - 1;
    if (found < 0) return {0, -1};
    const int end = __builtin_amdgcn_readlane(at, found + 1);
    if (end <= token) return {0, -1};
    s = base + found;
    len = __builtin_amdgcn_readlane(length, found);
    behind = (uint32_t)end - (uint32_t)token;
  } else {
    len = *(ScalarLoad)(a.context_lens + s);
  }
  const int L = min(max(len, 0), a.max_ctx);
  const int position = (int)((uint32_t)L - behind);
  return {s, behind <= (uint32_t)L ? position : -1};
}

// A workgroup has kPasses times kRows rows of a token.  They are all asked for before its position is looked up.
template <int kD, int kFormat, int kPasses>
__global__ __launch_bounds__(kThreads) void kv_rope_kernel(RopeLaunch a) {
  constexpr bool kFp4 = kFormat == kFp4Pools;
  constexpr int kLanes = kD / 8;            // of a row
  constexpr int kRows = kThreads / kLanes;  // at a time
  const int token = blockIdx.x;
  const int n = threadIdx.x & (kLanes - 1);
  const int rows = a.Hq + 2 * a.Hkv;
  const int row0 = blockIdx.y * kPasses * kRows + threadIdx.x / kLanes;

  // Where a lane's pieces begin: in a query or key, and in a value.  Tiles want eight dims in a row.
  const int half = a.R >> 1, split = a.R || kFp4 ? half : kD / 2;
  const bool turned = 8 * n < a.R, apart = !a.interleaved && 4 * n < split;
  const int p0 = apart ? 4 * n : 8 * n, p1 = apart ? split + 4 * n : 8 * n + 4;
  const int v0 = kFp4 ? 8 * n : 4 * n, v1 = kFp4 ? 8 * n + 4 : kD / 2 + 4 * n;
  Raw raw[kPasses];
  const uint16_t* const q = a.q + token * a.q_stride;
  const uint16_t* const k = a.k + token * a.k_stride - a.Hq * kD;
  const uint16_t* const v = a.v + token * a.v_stride - (a.Hq + a.Hkv) * kD;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int r = min(row0 + i * kRows, rows - 1);
    const bool is_v = r >= a.Hq + a.Hkv;
    raw[i] = load((is_v ? v : r >= a.Hq ? k : q) + r * kD, is_v ? v0 : p0, is_v ? v1 : p1);
  }
  Raw q_norm = {}, k_norm = {};
  if (a.q_norm) q_norm = load(a.q_norm, p0, p1);
  if (a.k_norm) k_norm = load(a.k_norm, p0, p1);

  const TokenAt at = token_at(a, token);
  if (at.position < 0) return;
  f32x4 cs = {}, sn = {};
  if (turned) {
    const float* row = a.cos_sin + (int64_t)at.position * a.R + 4 * n;
    cs = *(const f32x4*)row;
    sn = *(const f32x4*)(row + half);
  }
  const int id = a.block_tables[(int64_t)at.request * a.MAXB + (at.position >> a.log_block)];
  const bool mapped = (unsigned)id < (unsigned)a.NB;   // never follow a corrupt id; report it once per token
  if (!mapped && a.id_faults && blockIdx.y == 0 && threadIdx.x == 0) atomicAdd(a.id_faults, 1);
  const int slot = at.position & ((1 << a.log_block) - 1);

#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    __builtin_amdgcn_sched_barrier(0);   // one after the other: all at once takes three times the registers, and the workgroups on a unit hide the rest
    const int r = row0 + i * kRows;
    if (r >= rows) break;
    const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv;
    float x[8];
    unpack(raw[i], x);
    if (!is_v) {
      if (is_q ? a.q_norm : a.k_norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
#pragma unroll
        for (int m = 1; m < kLanes; m <<= 1) sum += __shfl_xor(sum, m);
        const float inv = __builtin_amdgcn_rsqf(sum * (1.f / kD) + a.eps);   // within a unit in the last place
        float w[8];
        unpack(is_q ? q_norm : k_norm, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * w[e];
      }
      if (!turned) {   // as they are: an infinity times a sine of zero would be none
      } else if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float one = x[2 * e], two = x[2 * e + 1];
          x[2 * e] = one * cs[e] - two * sn[e];
          x[2 * e + 1] = two * cs[e] + one * sn[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float one = x[e], two = x[4 + e];
          x[e] = one * cs[e] - two * sn[e];
          x[4 + e] = two * cs[e] + one * sn[e];
        }
      }
    }
    if (is_q) {
      put_bf16((char*)(a.q_out + ((int64_t)token * a.Hq + r) * kD), p0, p1, x);
    } else if (mapped) {
      const int head = is_v ? r - a.Hq - a.Hkv : r - a.Hq;
      const int64_t units = ((int64_t)id * a.Hkv + head) << (a.log_block - 4);
      char* pool = (char*)(is_v ? a.v_pool : a.k_pool);
      if constexpr (kFp4) {
        if (!is_v && half && !a.interleaved) {
          // the pieces that hold this lane's eight dims in a row, out of the lanes that have them
          float y[8];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int d = 8 * n + 4 * z;
            const bool low = d < half, high = !low && d < a.R;
            const int from = low ? d >> 2 : high ? (d - half) >> 2 : n;
            const bool second = high || (!low && z == 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float one = __shfl(x[e], from, kLanes), two = __shfl(x[4 + e], from, kLanes);
              y[4 * z + e] = second ? two : one;
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = y[e];
        }
        put_fp4<kD>(pool + (units + (slot >> 4)) * fp4_tile_bytes(kD), slot & 15, n, x, is_v);
      } else if constexpr (kFormat == 1) {
        char* row = pool + (units * kBlockTokens + slot) * kD;
        put_fp8(row, is_v ? v0 : p0, is_v ? v1 : p1, x, is_v ? a.v_scale : a.k_scale, is_v ? a.v_inverse : a.k_inverse);
      } else {
        put_bf16(pool + (units * kBlockTokens + slot) * kD * 2, is_v ? v0 : p0, is_v ? v1 : p1, x);
      }
    }
  }
}

template <int kD, int kPasses>
void launch_passes(const RopeLaunch& a, hipStream_t stream) {
  constexpr int kRows = kPasses * (kThreads / (kD / 8));
  const dim3 grid(a.T, (a.Hq + 2 * a.Hkv + kRows - 1) / kRows);
  if (a.kv_fp8 == kFp4Pools) hipLaunchKernelGGL((kv_rope_kernel<kD, kFp4Pools, kPasses>), grid, dim3(kThreads), 0, stream, a);
  else if (a.kv_fp8) hipLaunchKernelGGL((kv_rope_kernel<kD, 1, kPasses>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((kv_rope_kernel<kD, 0, kPasses>), grid, dim3(kThreads), 0, stream, a);
}
// Few tokens: as many workgroups as their rows give.  Many: up to four rows a lane, for which a position is looked up once (us at one, two and
// four, the kernel before lanes had both halves of a rotation: 16 prompts of 100..2000 tokens on 40/8 heads 142 / 113 / 105, at D = 256 256 / 218 / 200;
// 24 pieces of 1..900 in e4m3 on 32/8 heads at D = 64, of which two are all, 32 / 27).
template <int kD>
void launch_dim(const RopeLaunch& a, hipStream_t stream) {
  const int rows = a.Hq + 2 * a.Hkv, at_a_time = kThreads / (kD / 8);
  if (a.T < 1024 || rows <= at_a_time) launch_passes<kD, 1>(a, stream);
  else if (rows <= 2 * at_a_time) launch_passes<kD, 2>(a, stream);
  else launch_passes<kD, 4>(a, stream);
}

}  // namespace

hipError_t launch_kv_rope(const RopeLaunch& a, hipStream_t stream) {
  if (a.D == 64) launch_dim<64>(a, stream);
  else if (a.D == 128) launch_dim<128>(a, stream);
  else if (a.D == 256) launch_dim<256>(a, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
