// New tokens on their way into the cache, for gfx950: queries and keys normalised head by head and rotated to their positions, queries to
// the attention's input, keys and values to their slots of the paged pools, in one pass over the rows that a fused projection gives.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          a row of D values, where there are weights
//   (a, b) -> (a cos - b sin, b cos + a sin)    pairs (j, j + R/2) or (2j, 2j + 1) of the first R dims; cos and sin from the position's row
//
// in fp32, rounded once to what is stored.  A lane has eight dims of a row, D / 8 lanes a row, so the sum of squares and the partners of a
// rotation stay within 8 to 32 lanes.
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
__device__ __forceinline__ void unpack(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float to_range(float y) {
  return (y != y) ? y : fminf(fmaxf(y, -448.f), 448.f);   // NaN stays NaN
}

// Where eight dims of token t of 16, `chunk` of their KV head's row, go in its pool; `unit` is the first byte of the KV head's 16 tokens.
template <int kD>
__device__ __forceinline__ void put_bf16(char* unit, int t, int chunk, const float (&y)[8]) {
  *(u32x4*)(unit + (t * kD + 8 * chunk) * 2) = u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
}
// Divided by the pool's scale, clamped to the format's range and rounded to nearest even by the hardware conversion.
template <int kD>
__device__ __forceinline__ void put_fp8(char* unit, int t, int chunk, const float (&y)[8], float scale) {
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = to_range(y[i] / scale);
  u32x2 b;
  b.x = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false), true);
  b.y = __builtin_amdgcn_cvt_pk_fp8_f32(z[6], z[7], __builtin_amdgcn_cvt_pk_fp8_f32(z[4], z[5], 0, false), true);
  *(u32x2*)(unit + t * kD + 8 * chunk) = b;
}
// The scale of a group of 32 dims, which are four lanes', is the smallest power of two with which none is rounded past 6: 4 to 7 of it are in
// the largest.  Between 2^-120 and 2^125, so that no product with a code leaves the range of normal numbers.  The hardware's conversion
// rounds to nearest even and holds what is larger at 6; NaN is in the scale.
template <int kD>
__device__ __forceinline__ void put_fp4(char* unit, int t, int chunk, const float (&y)[8], bool is_v) {
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
    *(uint32_t*)(unit + fp4_k_place(chunk, t)) = w;
  } else if constexpr (kD == 64) {
    *(uint16_t*)(unit + fp4_v_place(kD, 8 * chunk, t)) = (uint16_t)w;
    *(uint16_t*)(unit + fp4_v_place(kD, 8 * chunk + 4, t)) = (uint16_t)(w >> 16);
  } else {
    *(uint32_t*)(unit + fp4_v_place(kD, 8 * chunk, t)) = w;
  }
  if ((chunk & 3) == 0) *(uint8_t*)(unit + fp4_scale_place(kD, chunk >> 2, t)) = most > 0x7f800000u ? 255 : byte;
}

// A token's request and position; position < 0: it has none.
struct TokenAt {
  int request, position;
};
__device__ __forceinline__ TokenAt token_at(const RopeLaunch& a, int token) {
  typedef const int32_t __attribute__((address_space(4))) * ScalarLoad;
  int s = token;
  uint32_t behind = 1;   // tokens of the request from this one on
  if (a.token_starts) {
    // the last request that begins at or before the token: two looks of 64 lanes, kMaxSeqs being 32 times 64
    const int lane = threadIdx.x & 63, step = (a.S + 63) >> 6;
    const int i = lane * step;
    const int begin = i < a.S ? a.token_starts[i] : INT32_MAX;
    const int base = (__popcll(__ballot(begin <= token)) - 1) * step;
    if (base < 0) return {0, -1};
    const int j = base + lane;
    const int at = lane < step && j < a.S ? a.token_starts[j] : INT32_MAX;
    s = __builtin_amdgcn_readfirstlane(min(max(base + __popcll(__ballot(at <= token)) - 1, 0), a.S - 1));
    const int end = *(ScalarLoad)(a.token_starts + s + 1);
    if (end <= token) return {0, -1};
    behind = (uint32_t)end - (uint32_t)token;
  }
  const int L = min(max(*(ScalarLoad)(a.context_lens + s), 0), a.max_ctx);
  const int position = (int)((uint32_t)L - behind);
  return {s, behind <= (uint32_t)L ? position : -1};
}

// A workgroup for a token, or several that have its rows in turn.
template <int kD, int kFormat>
__global__ __launch_bounds__(kThreads) void kv_rope_kernel(RopeLaunch a) {
  constexpr int kLanes = kD / 8;            // of a row
  constexpr int kRows = kThreads / kLanes;  // at a time
  const int token = blockIdx.x;
  const int chunk = threadIdx.x & (kLanes - 1);
  const int rows = a.Hq + 2 * a.Hkv;
  const TokenAt at = token_at(a, token);
  if (at.position < 0) return;
  const int half = a.R >> 1;
  const bool turned = 8 * chunk < a.R;
  const bool upper = !a.interleaved && 8 * chunk >= half;   // the second of its pairs
  // the partner's chunk: of the same row, R / 2 dims further on or back
  const int partner = !turned || a.interleaved ? chunk : upper ? chunk - (half >> 3) : chunk + (half >> 3);
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  if (turned) {
    const float* row = a.cos_sin + (int64_t)at.position * a.R;
    if (a.interleaved) {
      const f32x4 c4 = *(const f32x4*)(row + 4 * chunk), s4 = *(const f32x4*)(row + half + 4 * chunk);
#pragma unroll
      for (int i = 0; i < 8; ++i) { cs[i] = c4[i >> 1]; sn[i] = i & 1 ? s4[i >> 1] : -s4[i >> 1]; }
    } else {
      const int j = 8 * chunk - (upper ? half : 0);
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const f32x4 c4 = *(const f32x4*)(row + j + i), s4 = *(const f32x4*)(row + half + j + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) { cs[i + e] = c4[e]; sn[i + e] = upper ? s4[e] : -s4[e]; }
      }
    }
  }
  const int id = a.Hkv ? a.block_tables[(int64_t)at.request * a.MAXB + (at.position >> a.log_block)] : 0;
  const bool mapped = (unsigned)id < (unsigned)a.NB;   // never follow a corrupt id; report it once per token
  if (!mapped && a.id_faults && blockIdx.y == 0 && threadIdx.x == 0) atomicAdd(a.id_faults, 1);
  const int slot = at.position & ((1 << a.log_block) - 1);

  for (int r = blockIdx.y * kRows + threadIdx.x / kLanes; r < rows; r += gridDim.y * kRows) {
    const int kind = r < a.Hq ? 0 : r < a.Hq + a.Hkv ? 1 : 2;
    const int head = r - (kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hkv);
    const uint16_t* from = (kind == 0 ? a.q + token * a.q_stride : kind == 1 ? a.k + token * a.k_stride : a.v + token * a.v_stride) + head * kD;
    const u32x4 raw = *(const u32x4*)(from + 8 * chunk);
    float x[8];
    unpack(raw, x);
    if (kind < 2) {
      const uint16_t* norm = kind == 0 ? a.q_norm : a.k_norm;
      u32x4 other = raw;   // the partner's
      if (!a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__shfl((int)raw[i], partner, kLanes);
      }
      float y[8];
      unpack(other, y);
      if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
#pragma unroll
        for (int m = 1; m < kLanes; m <<= 1) sum += __shfl_xor(sum, m);
        const float inv = 1.f / sqrtf(sum * (1.f / kD) + a.eps);
        float w[8], wy[8];
        unpack(*(const u32x4*)(norm + 8 * chunk), w);
        unpack(*(const u32x4*)(norm + 8 * partner), wy);
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i] = x[i] * inv * w[i]; y[i] = y[i] * inv * wy[i]; }
      }
      if (turned) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = x[i] * cs[i] + (a.interleaved ? x[i ^ 1] : y[i]) * sn[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = z[i];
      }
    }
    if (kind == 0) {
      put_bf16<kD>((char*)(a.q_out + ((int64_t)token * a.Hq + head) * kD), 0, chunk, x);
    } else if (mapped) {
      const int64_t units = ((int64_t)id * a.Hkv + head) << (a.log_block - 4);
      char* pool = (char*)(kind == 1 ? a.k_pool : a.v_pool);
      if constexpr (kFormat == kFp4Pools) {
        put_fp4<kD>(pool + (units + (slot >> 4)) * fp4_tile_bytes(kD), slot & 15, chunk, x, kind == 2);
      } else if constexpr (kFormat == 1) {
        put_fp8<kD>(pool + units * (kBlockTokens * kD), slot, chunk, x, kind == 1 ? a.k_scale : a.v_scale);
      } else {
        put_bf16<kD>(pool + units * (kBlockTokens * kD * 2), slot, chunk, x);
      }
    }
  }
}

template <int kD>
void launch_dim(const RopeLaunch& a, hipStream_t stream) {
  const int rows = a.Hq + 2 * a.Hkv, at_a_time = kThreads / (kD / 8);
  const int passes = (rows + at_a_time - 1) / at_a_time;
  const dim3 grid(a.T, a.T < 1024 ? passes : 1);
  if (a.kv_fp8 == kFp4Pools) hipLaunchKernelGGL((kv_rope_kernel<kD, kFp4Pools>), grid, dim3(kThreads), 0, stream, a);
  else if (a.kv_fp8) hipLaunchKernelGGL((kv_rope_kernel<kD, 1>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((kv_rope_kernel<kD, 0>), grid, dim3(kThreads), 0, stream, a);
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
