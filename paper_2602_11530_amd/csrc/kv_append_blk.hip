// New tokens into e4m3 pools with a scale for each block and KV head, for gfx950.
//
//   scale 2^e, e the least from -117 to 119 with no |x| > 448 * 2^e among the call's values of a block and KV head; a block that held tokens keeps a
//   larger one, and if its own is smaller the rows that it held are rounded to 2^e;  byte = e4m3(x / scale)
//
// Scales are powers of two: dividing by one is exact, so that a value is rounded once, and again only where a block's scale grows past its subnormal
// ones.  The rows of a block and KV head, of K or of V, are one group of lanes' own, D / 8 lanes to a row, which turn them (kv_rope.h), find the largest
// among them without leaving registers, and write: no workgroup waits for another, nothing is read twice.  A scale's byte is read by all lanes of the
// group and written by one: where those are several wavefronts, behind the barrier at which they compare.
//
// Bound by memory: sixteen prompts of 100..2000 tokens on 40/8 heads (470 MB read and written) 91 us, 5.2 TB/s, 26 of them for K and V and 53 for the
// queries in the trace; pieces at D = 64 in 64-token blocks 27 us, 3.9 TB/s.  A step is one chain of loads, 2.8 us for 4 requests and 4.4 to 4.8 for 64
// where no scale grows.  Where some do, the rows that such a block held follow one after the other: with normal values 35 of 1024 blocks and heads of 64
// requests in 16-token blocks, and the step takes 8.6 us; 25 in 32-token blocks and 12.3; 16 in 64-token blocks and 19.3.
//   Rows spread over groups of lanes, at most 8 to a lane, all 8 asked for at once: with one group for a block, which takes its rows one after the
//   other and reads them twice, prompts took 102 us and pieces 59.
#include "kv_rope.h"

namespace pkv {
namespace {

// Slots: request s has slots token_starts[s] / B + 2 * s and on, which are enough wherever its tokens begin in a block.  For all lanes the same.
__device__ __forceinline__ InBlock in_block(const RopeLaunch& a, int slot) {
  typedef const int32_t __attribute__((address_space(4))) * ScalarLoad;
  int s = slot, start = slot, end = slot + 1, k = 0;
  if (a.token_starts) {
    // one look of 64 lanes up to 63 requests, else two, kMaxSeqs being 32 times 64
    const int lane = threadIdx.x & 63, step = (a.S >> 6) + 1;
    auto begin = [&](int i) { return min(max(a.token_starts[min(i, a.S)], 0), a.T); };
    int base = 0;
    if (step > 1) {
      const int i = lane * step;
      base = max(__popcll(__ballot(i < a.S && (begin(i) >> a.log_block) + 2 * i <= slot)) - 1, 0) * step;
    }
    const int j = base + lane, at = begin(j);
    const int found = __popcll(__ballot(j < a.S && lane < 63 && (at >> a.log_block) + 2 * j <= slot)) - 1;
    if (found < 0) return {0, 0, 0, 0};
    s = base + found;
    start = __builtin_amdgcn_readlane(at, found);
    end = __builtin_amdgcn_readlane(at, found + 1);
    k = slot - (start >> a.log_block) - 2 * s;
  }
  return tokens_in_block(s, start, end, min(max(*(ScalarLoad)(a.context_lens + s), 0), a.max_ctx), k, a.log_block);
}

__device__ __forceinline__ int pack_e4m3(float w, float x, float y, float z) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(y, z, __builtin_amdgcn_cvt_pk_fp8_f32(w, x, 0, false), true);
}

constexpr int kMany = 1024;   // tokens: each has work for a workgroup of its own

struct Scales {
  uint8_t *k, *v;
};

// Workgroups [0, append_groups): `parts` to a slot.  D / 8 lanes have a row, `spread` times that the rows of a block and KV head, which are keys of all heads
// and then values.  Those behind them, in a step's launch, have the queries: `q_parts` to a token.
// kHeld: rows of a block that a lane has at most, as it turned them.
template <int kD, int kHeld, int kQueries>
__global__ __launch_bounds__(kThreads) void kv_append_blk_kernel(RopeLaunch a, Scales scales, int spread, int parts, int append_groups, int q_parts) {
  typedef Lane<kD, 1> L;
  constexpr int kLanes = L::kLanes;
  __shared__ uint32_t most_of[kThreads / 64];   // of each wavefront, where a head's rows are more than one's
  const L lane(a);
  const int group = threadIdx.x / kLanes;
  if constexpr (kQueries > 0) if ((int)blockIdx.x >= append_groups) {
    const int at = blockIdx.x - append_groups, token = at / q_parts, rows = blockDim.x / kLanes;
    const int row0 = (at - token * q_parts) * kQueries * rows + group;
    Raw raw[kQueries];
#pragma unroll
    for (int i = 0; i < kQueries; ++i) raw[i] = lane.ask(a, token, min(row0 + i * rows, a.Hq - 1));
    asm volatile("" : : : "memory");   // all of them go out here, none only where it is used
    const TokenAt t = token_at(a, token);
    if (t.position < 0) return;
    f32x4 cs = {}, sn = {};
    lane.ask_turn(a, t.position, cs, sn);
#pragma unroll
    for (int i = 0; i < kQueries; ++i) {
      __builtin_amdgcn_sched_barrier(0);   // one after the other
      const int r = row0 + i * rows;
      if (r >= a.Hq) break;
      lane.finish(a, token, r, t.position, 0, raw[i], cs, sn);
    }
    return;
  }
  const int slot = blockIdx.x / parts, part = blockIdx.x - slot * parts;
  const InBlock at = in_block(a, slot);
  const int count = at.to - at.from;
  if (count <= 0) return;
  const int id = a.block_tables[(int64_t)at.s * a.MAXB + (at.from >> a.log_block)];
  if ((unsigned)id >= (unsigned)a.NB) {   // never follow a corrupt id
    if (part == 0 && threadIdx.x == 0 && a.id_faults) atomicAdd(a.id_faults, 1);
    return;
  }
  const int kinds = blockDim.x / (kLanes * spread);
  const int kind = part * kinds + group / spread, mine = group % spread;
  const bool live = kind < 2 * a.Hkv;
  const int of = min(kind, 2 * a.Hkv - 1);   // lanes without a head go along
  const bool is_v = of >= a.Hkv;
  const int head = is_v ? of - a.Hkv : of;
  const int slot0 = at.from & ((1 << a.log_block) - 1);   // rows before it were there
  uint8_t* scale_at = (is_v ? scales.v : scales.k) + (int64_t)id * scale_row_bytes(a.Hkv) + head;
  char* block = (char*)(is_v ? a.v_pool : a.k_pool) + (((int64_t)id * a.Hkv + head) << a.log_block) * kD;
  const int held = slot0 ? *scale_at : 0;

  // this lane's rows: `mine`, `mine` + spread and on, at most kHeld of them
  float x[kHeld][8];
  {
    Raw raw[kHeld];
    f32x4 cs[kHeld] = {}, sn[kHeld] = {};
#pragma unroll
    for (int i = 0; i < kHeld; ++i) raw[i] = lane.ask(a, at.token + min(mine + i * spread, count - 1), a.Hq + of);
    if (!is_v) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) lane.ask_turn(a, at.from + min(mine + i * spread, count - 1), cs[i], sn[i]);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) lane.template finish<true>(a, 0, a.Hq + of, 0, 0, raw[i], cs[i], sn[i], &x[i]);
  }
  // The largest of the magnitudes' bits, whose order is the numbers'.  Not by v_max_f32: what is neither normalised nor rotated is as it was in memory, and of
  // a signalling NaN that instruction makes a quiet one, instead of leaving it out (1 % of an append's time).
  auto size = [&](int i, int e) __attribute__((always_inline)) { return __float_as_uint(x[i][e]) & 0x7fffffffu; };
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
#pragma unroll
    for (int e = 0; e < 8; e += 2) most = max(max(most, size(i, e)), size(i, e + 1));
  const bool no_numbers = most >= 0x7f800000u;   // some are infinite or NaN, which do not count
  if (__builtin_expect(no_numbers, 0)) {
    most = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, size(i, e) < 0x7f800000u ? size(i, e) : 0u);
  }
  const int lanes = kLanes * spread;
  for (int step = 1; step < min(lanes, 64); step <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, step));
  if (lanes > 64) {
    if ((threadIdx.x & 63) == 0) most_of[threadIdx.x >> 6] = most;
    __syncthreads();
    const int first = threadIdx.x / lanes * (lanes / 64);
    for (int w = 0; w < lanes / 64; ++w) most = max(most, most_of[first + w]);
  }
  if (!live) return;
  // 448 is 1.75 * 2^8
  const int need = min(max((int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u), 10), 246), byte = max(held, need);
  if (slot0 && byte > held) {
    // what the block held, rounded to the larger scale; factors below 2^-100 leave zeros as that does
    const float factor = __uint_as_float((uint32_t)(127 - min(byte - held, 100)) << 23);
    for (int t = mine; t < slot0; t += spread) {
      u32x2* row = (u32x2*)(block + t * kD + 8 * lane.n);
      const u32x2 w = *row;
      u32x2 y;
#pragma unroll
      for (int z = 0; z < 2; ++z)
        y[z] = pack_e4m3(__builtin_amdgcn_cvt_f32_fp8(w[z], 0) * factor, __builtin_amdgcn_cvt_f32_fp8(w[z], 1) * factor,
                         __builtin_amdgcn_cvt_f32_fp8(w[z], 2) * factor, __builtin_amdgcn_cvt_f32_fp8(w[z], 3) * factor);
      *row = y;
    }
  }
  if (mine == 0 && lane.n == 0 && (!slot0 || byte != held)) *scale_at = (uint8_t)byte;
  const bool beyond = __any(no_numbers || need == 246);   // else no value is
  const float inverse = __builtin_ldexpf(1.f, 127 - byte);   // a subnormal number for a byte of 254, which was there
  const int p0 = choose(is_v, lane.v0, lane.p0), p1 = choose(is_v, lane.v1, lane.p1);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int t = mine + i * spread;
    if (t >= count) break;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[i][e] * inverse;
    if (beyond) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = to_range(y[e]);
    }
    char* row = block + (slot0 + t) * kD;
    __builtin_nontemporal_store(pack_e4m3(y[0], y[1], y[2], y[3]), (int*)(row + p0));
    __builtin_nontemporal_store(pack_e4m3(y[4], y[5], y[6], y[7]), (int*)(row + p1));
  }
}

template <int kD, int kHeld, int kQueries>
hipError_t launch_queries(const RopeLaunch& a, const Scales& scales, hipStream_t stream) {
  constexpr int kLanes = kD / 8;
  // a step has one row of a block, a prompt all of them
  const int spread = a.token_starts ? (1 << a.log_block) / kHeld : 1, lanes = kLanes * spread;
  const int all_lanes = 2 * a.Hkv * lanes, threads = all_lanes < kThreads && a.T < kMany ? (all_lanes + 63) / 64 * 64 : kThreads;
  const int kinds = threads / lanes, parts = (2 * a.Hkv + kinds - 1) / kinds;
  const int rows = kQueries * (threads / kLanes), q_parts = kQueries ? (a.Hq + rows - 1) / rows : 0;
  const int slots = a.token_starts ? (a.T >> a.log_block) + 2 * a.S : a.S;
  const int64_t append_groups = (int64_t)slots * parts, all = append_groups + (int64_t)a.T * q_parts;
  if (all * threads > UINT32_MAX) return hipErrorInvalidValue;   // a launch has fewer lanes
  hipLaunchKernelGGL((kv_append_blk_kernel<kD, kHeld, kQueries>), dim3((unsigned)all), dim3(threads), 0, stream, a, scales, spread, parts,
                     (int)append_groups, q_parts);
  return hipGetLastError();
}

template <int kD>
hipError_t launch_dim(const RopeLaunch& a, const Scales& scales, hipStream_t stream) {
  if (!a.token_starts) return a.q_out ? launch_queries<kD, 1, 1>(a, scales, stream) : launch_queries<kD, 1, 0>(a, scales, stream);
  if (!a.q_out) return launch_queries<kD, 8, 0>(a, scales, stream);
  if (a.T < kMany) return launch_queries<kD, 8, 1>(a, scales, stream);
  // many queries by themselves: beside rows that are held they have half the wavefronts that hide their loads (94 us as one launch 106)
  const hipError_t e = launch_queries<kD, 8, 0>(a, scales, stream);
  if (e != hipSuccess) return e;
  RopeLaunch rest = a;
  rest.Hkv = 0;
  rest.kv_fp8 = 1;
  rest.id_faults = nullptr;
  return launch_kv_rope(rest, stream);
}

}  // namespace

hipError_t launch_kv_append_blk(const RopeLaunch& a, uint8_t* k_scales, uint8_t* v_scales, hipStream_t stream) {
  const Scales scales = {k_scales, v_scales};
  if (a.D == 64) return launch_dim<64>(a, scales, stream);
  if (a.D == 128) return launch_dim<128>(a, scales, stream);
  if (a.D == 256) return launch_dim<256>(a, scales, stream);
  return hipErrorInvalidValue;
}

}  // namespace pkv
