// New tokens on their way into the cache, for gfx950: queries and keys normalised head by head and rotated to their positions, queries to
// the attention's input, keys and values to their slots of the paged pools, in one pass over the rows that a fused projection gives.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          a row of D values, where there are weights
//   (a, b) -> (a cos - b sin, b cos + a sin)    pairs (j, j + R/2) or (2j, 2j + 1) of the first R dims; cos and sin from the position's row
//
// in fp32, rounded once to what is stored.  Prompts are bound by memory, each row in and out once (16 of 100..2000 tokens on 40/8 heads, 505 MB,
// 86 us: 5.9 TB/s, a 1 GiB copy 4.8), a step's few tokens by the launch and three round trips: lengths, the position's row and table entry,
// stores.  D / 8 lanes have a row, and a lane two pieces of four dims: with pairs (j, j + R/2) those of both
// halves, so that a rotation stays in the lane, else (and behind the first R dims) eight in a row.  Into bf16 and e4m3 pools the sum of squares is all
// that lanes exchange; tiles want a key's dims eight in a row, which are taken from the lanes that have them, and the largest of a group of 32, which is
// four lanes' (the prompts above 89 us, 453 MB).
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
  // A row that has arrived, to where it belongs; `id`: the block of its position.
  __device__ __forceinline__ void finish(const RopeLaunch& a, int64_t token, int r, int position, int id, const Raw& raw, const f32x4& cs,
                                         const f32x4& sn) const {
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

// Reports a refused id, once per token.
__device__ __forceinline__ void report(const RopeLaunch& a, int id) {
  if ((unsigned)id >= (unsigned)a.NB && a.id_faults) atomicAdd(a.id_faults, 1);
}

// A workgroup has kPasses times kRows rows of a token.  They are all asked for before its position is looked up.
template <int kD, int kFormat, int kPasses>
__global__ __launch_bounds__(kThreads) void kv_rope_kernel(RopeLaunch a) {
  typedef Lane<kD, kFormat> L;
  const int token = blockIdx.x, rows = a.Hq + 2 * a.Hkv;
  const int row0 = blockIdx.y * kPasses * L::kRows + threadIdx.x / L::kLanes;
  const L lane(a);
  Raw raw[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) raw[i] = lane.ask(a, token, min(row0 + i * L::kRows, rows - 1));
  asm volatile("" : : : "memory");   // all of them go out here, none only where it is used
  const TokenAt at = token_at(a, token);
  if (at.position < 0) return;
  f32x4 cs = {}, sn = {};
  lane.ask_turn(a, at.position, cs, sn);
  const int id = a.block_tables[(int64_t)at.request * a.MAXB + (at.position >> a.log_block)];
  if (blockIdx.y == 0 && threadIdx.x == 0) report(a, id);
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    __builtin_amdgcn_sched_barrier(0);   // one after the other: all at once takes three times the registers, and the workgroups on a unit hide the rest
    const int r = row0 + i * L::kRows;
    if (r >= rows) break;
    lane.finish(a, token, r, at.position, id, raw[i], cs, sn);
  }
}

// The rows of all tokens one after the other, where a token has few: a workgroup has kPasses times kRows of them, of several tokens.
template <int kD, int kFormat, int kPasses>
__global__ __launch_bounds__(kThreads) void kv_rope_rows_kernel(RopeLaunch a) {
  typedef Lane<kD, kFormat> L;
  const int rows = a.Hq + 2 * a.Hkv;
  const uint32_t from = blockIdx.x * (uint32_t)(kPasses * L::kRows);   // below T * rows, which is less than 2^24 * 32
  const int first = from / (uint32_t)rows, ahead = from - (uint32_t)first * rows;   // the first token, and its rows that others have
  const float per = __builtin_amdgcn_rcpf((float)rows);
  const L lane(a);
  Raw raw[kPasses];
  int token[kPasses], row[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int at = ahead + i * L::kRows + threadIdx.x / L::kLanes;
    const int t = (int)(((float)at + 0.5f) * per);   // a small quotient: (x + 1/2) / n is 1 / (2n) away from a whole number
    row[i] = at - t * rows;
    token[i] = first + t;
    raw[i] = lane.ask(a, min(token[i], a.T - 1), row[i]);
  }
  asm volatile("" : : : "memory");   // all of them go out here, none only where it is used
  const TokenAt begin = token_at(a, first);
  int position[kPasses], id[kPasses];
  f32x4 cs[kPasses] = {}, sn[kPasses] = {};
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    TokenAt at = begin;
    const int d = token[i] - first;
    if (d < begin.behind) at.position += d;
    else at = lane_token_at(a, min(token[i], a.T - 1));
    position[i] = token[i] < a.T && at.position >= 0 ? at.position : -1;
    id[i] = 0;
    if (position[i] >= 0) {
      id[i] = a.block_tables[(int64_t)at.request * a.MAXB + (position[i] >> a.log_block)];
      lane.ask_turn(a, position[i], cs[i], sn[i]);
    }
  }
  asm volatile("" : : : "memory");
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (position[i] < 0) continue;
    if (row[i] == 0 && lane.n == 0) report(a, id[i]);
    lane.finish(a, token[i], row[i], position[i], id[i], raw[i], cs[i], sn[i]);
  }
}

template <int kD, int kPasses, bool kTokens>
void launch_passes(const RopeLaunch& a, hipStream_t stream) {
  constexpr int kRows = kPasses * (kThreads / (kD / 8));
  const int rows = a.Hq + 2 * a.Hkv;
  const dim3 grid = kTokens ? dim3(a.T, (rows + kRows - 1) / kRows) : dim3((unsigned)(((int64_t)a.T * rows + kRows - 1) / kRows));
  const auto kernel = [&](auto format) {
    if constexpr (kTokens) return kv_rope_kernel<kD, decltype(format)::value, kPasses>;
    else return kv_rope_rows_kernel<kD, decltype(format)::value, kPasses>;
  };
  const auto k = a.kv_fp8 == kFp4Pools ? kernel(std::integral_constant<int, kFp4Pools>{})
                 : a.kv_fp8            ? kernel(std::integral_constant<int, 1>{})
                                       : kernel(std::integral_constant<int, 0>{});
  hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, stream, a);
}
// Few tokens: as many workgroups as their rows give.  Many: up to four rows a lane, for which a position is looked up once; where a token's rows
// do not fill a workgroup, rows of several tokens.  Us for 16 prompts of 100..2000 tokens: 40/8 heads 88, the rows in a row 111, at D = 256 176 /
// 208, 28/4 heads 66 / 72; 8/2 heads 27.8 / 23.7, 8/1 26.8 / 21.0, at D = 64 23.2 / 12.1, 16/8 there 30.5 / 28.6.
// Where many begins: us of the two ways for a step of 256, 512, 1000, 2000 requests, by replays of a graph (few / many): 40/8 heads 3.6 / 4.5, 4.7 / 5.1,
// 7.6 / 7.4, 12.8 / 11.0, tiles 4.0 / 4.6, 5.5 / 5.7, 8.3 / 8.4, 14.1 / 12.3; 32/8 at D = 64 3.1 / 3.5, 3.7 / 3.7, 4.7 / 4.5, 8.0 / 6.6; 16/8 at D = 256
// 3.6 / 4.6, 4.8 / 5.2, 7.8 / 7.9, 13.1 / 12.2; 8/1 2.9 / 4.0, 3.1 / 4.1, 3.6 / 4.3, 4.7 / 4.8.
template <int kD>
void launch_dim(const RopeLaunch& a, hipStream_t stream) {
  const int rows = a.Hq + 2 * a.Hkv, at_a_time = kThreads / (kD / 8);
  if (a.T < 1024) launch_passes<kD, 1, true>(a, stream);
  else if (rows <= at_a_time) launch_passes<kD, 2, false>(a, stream);
  else if (rows <= 2 * at_a_time) launch_passes<kD, 2, true>(a, stream);
  else launch_passes<kD, 4, true>(a, stream);
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
