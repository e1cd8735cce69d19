// New tokens' rows on their way into the cache: what the kernels that normalise, rotate and append them share.
#pragma once

#include "fp4.h"
#include "pkv_kernels.h"

#include <type_traits>

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
// By value: a choice between members of a struct would be one between their addresses, and the struct would live in memory.
__device__ __forceinline__ int choose(bool one, int x, int y) { return one ? x : y; }
__device__ __forceinline__ Raw choose(bool one, Raw x, Raw y) {
  return Raw{{one ? x.piece[0] : y.piece[0], one ? x.piece[1] : y.piece[1]}};
}
__device__ __forceinline__ Raw load(const uint16_t* row, int p0, int p1) { return Raw{{*(const u32x2*)(row + p0), *(const u32x2*)(row + p1)}}; }
__device__ __forceinline__ float to_range(float y) {
  return (y != y) ? y : fminf(fmaxf(y, -448.f), 448.f);   // NaN stays NaN
}

// A lane's pieces, which begin at dims p0 and p1, into a row; nontemporal, as nothing of a prompt is read again soon: 16 prompts of 100..2000 tokens on
// 40/8 heads 105 us with ordinary stores, 100 this way (of an earlier kernel), 24 pieces of 1..900 in e4m3 at D = 64 29.5 and 24.2; nontemporal loads
// gain nothing and cost 4 us where the projection's rows are still on chip.
__device__ __forceinline__ void put_bf16(char* row, int p0, int p1, const float (&y)[8]) {
  __builtin_nontemporal_store(u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])}, (u32x2*)(row + 2 * p0));
  __builtin_nontemporal_store(u32x2{pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])}, (u32x2*)(row + 2 * p1));
}
// Divided by the pool's scale, clamped to the format's range and rounded to nearest even by the hardware conversion.  `inverse`: the scale's
// rounded reciprocal, or 0.  With it a product and its remainder give the rounded quotient (Markstein's theorem) in three operations instead
// of ten, wherever the quotient is in range.  The remainder is taken as product less dividend: of a zero it is +0 for either sign, and less
// that a zero keeps its own, as a quotient does.
__device__ __forceinline__ void put_fp8(char* row, int p0, int p1, const float (&y)[8], float scale, float inverse) {
  float z[8];
  if (inverse != 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = y[i] * inverse, exact = __builtin_fmaf(-__builtin_fmaf(q, scale, -y[i]), inverse, q);
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

// A token's request and position (< 0: it has none), and how many tokens from it on are the request's.
struct TokenAt {
  int request, position, behind;
};
// `end`: where the request's tokens end; `len`: its context length.
__device__ __forceinline__ TokenAt placed(const RopeLaunch& a, int request, int token, int end, int len) {
  const int L = min(max(len, 0), a.max_ctx);
  const uint32_t behind = (uint32_t)end - (uint32_t)token;
  if (end <= token || behind > (uint32_t)L) return {0, -1, 1};
  return {request, (int)((uint32_t)L - behind), (int)behind};
}
// For all lanes the same.
__device__ __forceinline__ TokenAt token_at(const RopeLaunch& a, int token) {
  typedef const int32_t __attribute__((address_space(4))) * ScalarLoad;
  if (!a.token_starts) return placed(a, token, token, token + 1, *(ScalarLoad)(a.context_lens + token));
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
  if (found < 0) return {0, -1, 1};
  return placed(a, base + found, token, __builtin_amdgcn_readlane(at, found + 1), __builtin_amdgcn_readlane(length, found));
}
// Each lane's own.
__device__ __forceinline__ TokenAt lane_token_at(const RopeLaunch& a, int token) {
  if (!a.token_starts) return placed(a, token, token, token + 1, a.context_lens[token]);
  int s = -1;   // the last request that begins at or before the token
  for (int step = 1 << (31 - __clz(a.S)); step > 0; step >>= 1)
    if (s + step < a.S && a.token_starts[s + step] <= token) s += step;
  if (s < 0) return {0, -1, 1};
  return placed(a, s, token, a.token_starts[s + 1], a.context_lens[s]);
}

// What is a lane's of the rows it has: its pieces begin at p0 and p1 in a query or key, at v0 and v1 in a value (tiles want eight dims in a row).
template <int kD, int kFormat>
struct Lane {
  static constexpr bool kFp4 = kFormat == kFp4Pools;
  static constexpr int kLanes = kD / 8;             // of a row
  static constexpr int kRows = kThreads / kLanes;   // of a workgroup, at a time
  int n, half, p0, p1, v0, v1;
  bool turned;
  Raw q_norm, k_norm;
  __device__ __forceinline__ Lane(const RopeLaunch& a) {
    n = threadIdx.x & (kLanes - 1);
    half = a.R >> 1;
    turned = 8 * n < a.R;
    const int split = a.R || kFp4 ? half : kD / 2;
    const bool apart = !a.interleaved && 4 * n < split;
    p0 = apart ? 4 * n : 8 * n;
    p1 = apart ? split + 4 * n : 8 * n + 4;
    v0 = kFp4 ? 8 * n : 4 * n;
    v1 = kFp4 ? 8 * n + 4 : kD / 2 + 4 * n;
    q_norm = k_norm = Raw{};
    if (a.q_norm) q_norm = load(a.q_norm, p0, p1);
    if (a.k_norm) k_norm = load(a.k_norm, p0, p1);
  }
  // Row r of a token: its queries, its keys, its values.
  __device__ __forceinline__ Raw ask(const RopeLaunch& a, int64_t token, int r) const {
    const bool is_v = r >= a.Hq + a.Hkv;
    const uint16_t* row = is_v ? a.v + token * a.v_stride - (a.Hq + a.Hkv) * kD : r >= a.Hq ? a.k + token * a.k_stride - a.Hq * kD : a.q + token * a.q_stride;
    return load(row + r * kD, choose(is_v, v0, p0), choose(is_v, v1, p1));
  }
  __device__ __forceinline__ void ask_turn(const RopeLaunch& a, int position, f32x4& cs, f32x4& sn) const {
    if (!turned) return;
    const float* row = a.cos_sin + (int64_t)position * a.R + 4 * n;
    cs = *(const f32x4*)row;
    sn = *(const f32x4*)(row + half);
  }
  // A row that has arrived, normalised and rotated, to where it belongs; `id`: the block of its position.  kTurnOnly: to `turned_row`.
  template <bool kTurnOnly = false>
  __device__ __forceinline__ void finish(const RopeLaunch& a, int64_t token, int r, int position, int id, const Raw& raw, const f32x4& cs,
                                         const f32x4& sn, float (*turned_row)[8] = nullptr) const {
    const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv;
    float x[8];
    unpack(raw, x);
    if (!is_v) {
      if (is_q ? a.q_norm : a.k_norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
#pragma unroll
        for (int m = 1; m < kLanes; m <<= 1) sum += __shfl_xor(sum, m);
        const float mean = sum * (1.f / kD) + a.eps;
        // within a unit in the last place; the instruction takes subnormal numbers for zero
        const bool small = mean < 0x1p-126f;
        const float inv = __builtin_amdgcn_rsqf(small ? mean * 0x1p48f : mean) * (small ? 0x1p24f : 1.f);
        float w[8];
        unpack(choose(is_q, q_norm, k_norm), w);
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
    if constexpr (kTurnOnly) {
#pragma unroll
      for (int e = 0; e < 8; ++e) (*turned_row)[e] = x[e];
      return;
    }
    if (is_q) {
      put_bf16((char*)(a.q_out + (token * a.Hq + r) * kD), p0, p1, x);
      return;
    }
    if ((unsigned)id >= (unsigned)a.NB) return;   // never follow a corrupt id
    const int slot = position & ((1 << a.log_block) - 1), head = is_v ? r - a.Hq - a.Hkv : r - a.Hq;
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
      put_fp8(row, choose(is_v, v0, p0), choose(is_v, v1, p1), x, is_v ? a.v_scale : a.k_scale, is_v ? a.v_inverse : a.k_inverse);
    } else {
      put_bf16(pool + (units * kBlockTokens + slot) * kD * 2, choose(is_v, v0, p0), choose(is_v, v1, p1), x);
    }
  }
};

}  // namespace
}  // namespace pkv
