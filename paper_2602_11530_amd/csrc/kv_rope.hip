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
#include "kv_rope.h"

namespace pkv {
namespace {

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
