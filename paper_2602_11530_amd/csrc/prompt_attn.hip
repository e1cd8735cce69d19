// Causal attention of new tokens over the paged cache, for gfx950.
//
//   out[i, h] = sum_t softmax_t(scale * q[i, h] . K[t, h / G]) * V[t, h / G]     for t <= p_i, the position of token i
//
// A workgroup has the rows (token, head of the group) of some tokens of one request and KV head, 32 to a wavefront, 128 in all, and goes over the keys
// that the last of them sees, a tile of 32 or 64 at a time.  K and V of a tile are staged in LDS as bf16 once for all rows.  Per 32 keys, lane = 32*h + n:
//   S^T = K . Q^T   D/16 v_mfma_f32_32x32x16_bf16.  A = K rows, lane (n, h) has the 16 bytes at dims 16*jj + 8*h of key n; B = q, which stays in
//         registers, lane (n, h) has the same dims of row n.  The result leaves lane (n, h) with row n's scores of keys 8*(r / 4) + 4*h + r % 4.
//   P     = exp2(score - m), rounded to bf16.  A lane has scores of one row alone, so that maximum, sum and rescale stay in the lane but for one
//         exchange between the halves when the maximum is raised.
//   O^T  += V^T . P^T  D/32 times two for 32 keys.  P is the B operand as it came out; A takes dims in rows out of V's rows of dims by
//         transposing reads of LDS, four keys of 16 dims to 16 lanes, in the order of keys that P has.
// The running maximum is only raised when a score exceeds it by more than 2^8, as in the decode kernels.  A weight is one bf16 number here, off by
// 2^-8 of itself at most, while the decode kernels take two: the second is half as many matrix instructions again (one prompt of 8191 tokens 635 -> 860 us,
// sixteen of 100..2000 304 -> 385, at D = 256 130 -> 206), and many weights make up a row, so that rows are 0.0020 to 0.0023 from those in 64 bits (relative
// L2) where the rounding of the output alone makes 0.0016.  Few rows (kAlone) over bf16 pools wait for memory and have both numbers (4 tokens of each of 32
// requests 112.4 and 112.5 us), over 8-bit pools one (65 us, with two 71; at D = 64 67 and 75).
//
// Bound by the matrix unit and the vector unit together: 32 keys at D = 128 are 16 matrix instructions of 32 cycles and 90 vector ones, 16 of them
// exponentials, in one chain, so that the wavefronts of a SIMD have to cover each other.  The matrix unit is busy for 63 % of one prompt of 8191 tokens
// (40 heads on 8: 645 us, 1.06 PFLOP/s; a library product of 8192^3 reaches 1.21), for 45 % of sixteen of 100..2000 (303 us, 0.80), where a workgroup has
// some twenty tiles and its chain of loads before the first (arguments, starts, table, unit) is 3 us.
//   128 rows: LDS is read once for 32 rows and memory once for 128; the LDS unit is active for 23 to 45 % of the time.  One wavefront with 64 rows
//   has no registers left at D = 128; eight wavefronts were no faster.
//   Two tiles in LDS in turn, so that a tile's barrier is the only one.  Three: 664 -> 672 us.
//   bf16 goes from memory straight into LDS, where each lane asks for the piece whose place is its own: no registers in between, no stores to LDS.
//   e4m3 goes through registers, where it is widened once for all rows; at D = 256, where two workgroups to a unit leave no registers for it, it waits in
//   LDS as it is, behind a second barrier (e4m3 203 -> 156 us, eight prompts of 200..1500 tokens).
//   D = 256 in 256 registers, two workgroups to a unit, instead of one with 300: 194 -> 146 us.
//   Few rows (kAlone): where a request has rows for one wavefront, three would wait for it.  All four take them, each with every fourth tile, in LDS of its
//   own without barriers, nontemporal where nobody else reads it, and join in the end.  4 tokens of each of 32 requests with 1000..8000 behind them, memory's
//   case (592 MB): 125 -> 114 us (5.2 TB/s), 11 of them by the loads' kind; over e4m3 85 -> 64, of 200 requests 713 -> 636 (6.0 TB/s) and 448 -> 338.
//   Of a request with more rows the loads are ordinary: 255 single tokens beside 1200 behind 4000 1074 -> 901 us, with 128 rows to a workgroup 912.
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
constexpr float kTooLarge = 0x1p120f;              // a scale whose products with e4m3 values may not be finite
constexpr int kRawBuffer = 0x00020000;
constexpr int kMfma = 0x8, kDsRead = 0x100;       // kinds of instructions, for the scheduler

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kMaxPieces = 64;                    // of a context
// Keys of a tile, where contexts are cut and where they are whole.  With 32 at D = 128 three workgroups go on a unit instead of two: sixteen prompts of
// 100..2000 tokens 324 -> 298 us, over e4m3 335 -> 314; contexts that are cut stay long for their workgroups: 512 tokens behind 32000 371 us
// with 64 and 388 with 32.
__host__ __device__ constexpr int prompt_keys(int D, bool cut) { return D == 256 || (D == 128 && !cut) ? 32 : 64; }
// Workgroups that run on a compute unit at once, by their registers and LDS.
constexpr int prompt_groups(int D, int keys, bool alone) { return D == 64 ? 4 : alone ? 256 / D : D == 128 && keys == 32 ? 3 : 2; }

// A workgroup's tokens: `first` to `first + count` of the call, of request s, at position `at` and on.
struct Tokens {
  int s, first, count, at;
  bool only;   // the request's only ones
};
// The sum over the 64 lanes, the same for all: prefix sums of 16 lanes, then their last ones to the rows behind.
__device__ __forceinline__ int sum_of_lanes(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);   // row_bcast 15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);   // row_bcast 31
  return __builtin_amdgcn_readlane(x, 63);
}
// The x-th group of `per` tokens, those first whose tokens see most keys, of up to 64 requests: a lane has one.  A request's groups see `per` keys more each,
// so that it has one at each of some levels in a row, and those at or above a level are counted without a list of them.
__device__ __forceinline__ Tokens tokens_in_order(const PromptLaunch& a, int x, int per) {
  const int lane = threadIdx.x & 63, j = min(lane, a.S - 1);
  const int begin = min(max(a.token_starts[j], 0), a.T), end = min(max(a.token_starts[j + 1], 0), a.T);
  const int length = min(max(a.context_lens[j], 0), a.max_ctx);
  const int n = lane < a.S ? max(end - begin, 0) : 0;
  const int below = max(length - n, 0) / per, count = (n + per - 1) / per;     // its levels are below + 1 to below + count
  auto at_or_above = [&](int level) { return sum_of_lanes(min(max(below + count + 1 - level, 0), count)); };
  if (x >= sum_of_lanes(count)) return {0, 0, 0, 0, true};
  int level = 0, more = 0;        // the highest with more than x groups at or above it
  for (int step = 1 << (31 - __builtin_clz(a.max_ctx / per + a.T / per + 2)); step > 0; step >>= 1) {
    const int c = at_or_above(level + step);
    if (c > x) level += step;
    else more = c;
  }
  const bool has = below < level && level <= below + count;
  const uint64_t those = __ballot(has);
  const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(those >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)those, 0));
  const int s = __builtin_ctzll(__ballot(has && rank == x - more));
  const int from = __builtin_amdgcn_readlane(begin, s), tokens = __builtin_amdgcn_readlane(n, s), L = __builtin_amdgcn_readlane(length, s);
  const int slot = level - 1 - __builtin_amdgcn_readlane(below, s);
  const int lo = max(slot * per, max(tokens - L, 0)), hi = min((slot + 1) * per, tokens);
  return {s, from + lo, max(hi - lo, 0), L - tokens + lo, tokens <= per};
}
// Slots of `per` tokens: request s has slots start / per + s and on, one or none of them empty.
__device__ __forceinline__ Tokens tokens_of(const PromptLaunch& a, int slot, int per) {
  int s, from, end, L;
  if (!a.token_starts) {
    s = from = slot;
    end = from + 1;
    if (s >= a.S) return {0, 0, 0, 0, true};
    slot = 0;
    L = *(ScalarLoad)(a.context_lens + s);
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
    const int length = j < a.S ? a.context_lens[j] : 0;          // with the starts: one round trip less
    const int found = __popcll(__ballot(j < a.S && lane < 63 && at / per + j <= slot)) - 1;
    if (found < 0) return {0, 0, 0, 0, true};
    s = base + found;
    from = __builtin_amdgcn_readlane(at, found);
    end = __builtin_amdgcn_readlane(at, found + 1);
    slot -= from / per + s;
    L = __builtin_amdgcn_readlane(length, found);
  }
  L = min(max(L, 0), a.max_ctx);
  const int n = end - from;
  // tokens before position 0 have none
  const int skip = max(n - L, 0);
  const int lo = max(slot * per, skip), hi = min((slot + 1) * per, n);
  return {s, from + lo, max(hi - lo, 0), L - n + lo, n <= per};
}

__device__ __forceinline__ u32x2 widen(uint32_t w, float scale) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, true))};
}

// 64 lanes' pieces of a buffer, zeros out of its bounds, to 1 KiB in a row of LDS from `to` on.  An opaque instruction: the compiler would wait for it
// before every read of LDS that follows, whatever it reads.  Who asks waits for what was asked for, and meets the others, before anyone reads it.
// once: nobody else reads it, and it need not stay in the caches.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t b, uint32_t to, int offset, bool once) {
  if (once) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" : : "s"(to), "v"(offset), "s"(b) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to), "v"(offset), "s"(b) : "memory");
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

template <int kD, int kFormat, int kKeyTile, bool kAlone>
__global__ __launch_bounds__(kThreads, prompt_groups(kD, kKeyTile, kAlone)) void prompt_attn_kernel(PromptLaunch a, int per, int slots, uint32_t group_inverse) {
  constexpr int kSteps = kD / 16, kTiles = kD / 32;
  constexpr int kHalves = kKeyTile / 32;
  constexpr int kUnits = kKeyTile / kBlockTokens;                // of a tile
  constexpr int kWindowTiles = 64 / kUnits;                      // whose units a wavefront's lanes describe
  constexpr int kTileBytes = kKeyTile * kD * 2;
  constexpr int kElem = kFormat == 0 ? 2 : 1;
  constexpr int kSource = kKeyTile * kD * kElem / 16;            // 16-byte pieces of a tile as the pool has it
  constexpr int kLoads = kSource / (kAlone ? 64 : kThreads);     // of a lane
  constexpr int kPerToken = kD * kElem / 16;
  constexpr int kOfUnit = kPerToken * kBlockTokens;
  constexpr int kOwn = kAlone ? kUnits : 1, kEach = kLoads / kOwn;   // units that a wavefront loads from, its loads of one
  static_assert(kEach * kOwn * (kAlone ? 64 : kThreads) == kSource && kOfUnit % (64 * kEach) == 0, "whole units, or pieces of one");
  constexpr bool kDirect = kFormat == 0;                         // nothing to widen: from memory straight into LDS
  constexpr bool kTwo = kAlone && kFormat == 0;                  // weights are two bf16 numbers
  constexpr bool kStaged = kFormat != 0 && kD == 256 && !kAlone;            // on its way to registers through LDS
  constexpr bool kHide = kD > 64 && kKeyTile == 32 && !kAlone;              // registers are short: what is cheap to find again is not kept in one over the loop
  constexpr int kReadsAhead = kAlone ? 4 : kD == 256 ? 2 : kKeyTile == 32 ? 3 : 6;   // of LDS in the first product, as many as there are registers for
  // K and V of two tiles in turn, or of one as bf16 and behind it of the next as it is
  __shared__ __align__(16) char lds[kAlone ? 2 * kWaves * kTileBytes : kStaged ? 2 * kTileBytes + 32 * kSource : 4 * kTileBytes];
  __shared__ int first_bad[kD];                                  // the first key whose V is not finite there, of those that some row does not see
  __shared__ int any_bad;
  [[maybe_unused]] __shared__ float stats_of[kAlone ? kWaves : 1][2][32];   // kAlone: of a wavefront's rows

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int kvh = blockIdx.x % a.Hkv;
  const int slot = slots - 1 - (int)(blockIdx.x / a.Hkv);        // late tokens see most: they begin first
  const Tokens tok = !kAlone && a.ordered ? tokens_in_order(a, slots - 1 - slot, per) : tokens_of(a, slot, per);
  const int keys = tok.at + tok.count;                           // that the last one sees
  const int tiles = (keys + kKeyTile - 1) / kKeyTile;
  const int from = blockIdx.y * a.piece, to = min(from + a.piece, tiles);
  if (tok.count <= 0 || from >= to) return;

  // This lane's row, and the last key that it sees; rows behind the last are computed along with it.
  struct Row {
    int of_call, last_key;
    bool live;
  };
  auto row_of = [&](int lane) __attribute__((always_inline)) -> Row {
    const int row = (kAlone ? 0 : 32 * wave) + (lane & 31), which = (int)((row * group_inverse) >> 16), head = row - which * a.G;   // row / G, row % G
    const int at = min(which, tok.count - 1);
    return {(tok.first + at) * a.Hq + kvh * a.G + head, tok.at + at, which < tok.count};   // T * Hq is below 2^31
  };
  // With kHide the compiler does not know that this is the same number as before.
  auto again = [&](int& x) __attribute__((always_inline)) { if constexpr (kHide) asm volatile("" : "+v"(x)); };
  auto this_lane = [&]() __attribute__((always_inline)) -> int {
    int here = lane;
    again(here);
    return here;
  };
  const int last_key = row_of(lane).last_key;
  const int wave_from = __builtin_amdgcn_readlane(last_key, 0), wave_to = __builtin_amdgcn_readlane(last_key, 31);
  const bool idle = __builtin_amdgcn_readfirstlane(!__any(row_of(lane).live));

  bf16x8 q[kSteps];
  const bool negative = a.scale_log2e < 0.f;
  // masked scores stay -inf with a scale of zero, too; NaN stays NaN
  const float scale = __builtin_fabsf(a.scale_log2e) < 0x1p-126f ? 0x1p-126f : __builtin_fabsf(a.scale_log2e);
#pragma unroll
  for (int jj = 0; jj < kSteps; ++jj) {
    u32x4 x = *(const u32x4*)(a.q + (int64_t)row_of(lane).of_call * kD + 16 * jj + 8 * h);
    if (negative) x ^= 0x80008000u;
    q[jj] = __builtin_bit_cast(bf16x8, x);
  }

  // Units of the context: one to a lane, a window of 64 at a time and the next one ahead.  What a load needs of its unit is worked out there, 64 units
  // at a time, and read from the lane.
  struct Window {
    uint64_t at;    // of the unit's K, 16 keys of the KV head
    int scales;     // kBlkPools: of K, of V
    uint64_t gone;  // a bit for each unit that is not there
  };
  const int log_units = a.log_block - 4;
  const int context = tok.at + tok.count;   // keys behind this are not seen
  const uint64_t v_behind = (uint64_t)a.v_pool - (uint64_t)a.k_pool;   // of a unit's V behind its K
  int refused = 0;
  auto describe = [&](int tile) -> Window {
    const int u = kUnits * tile + lane;
    const bool here = u >= kUnits * from && u * kBlockTokens < context && u < kUnits * to;
    int id = -1;
    if (here) id = a.block_tables[(int64_t)tok.s * a.MAXB + (u >> log_units)];
    const bool mapped = (unsigned)id < (unsigned)a.NB;           // ids outside the pool are never followed
    refused += __popcll(__ballot(here && !mapped));
    Window w;
    const int slab = mapped ? ((id * a.Hkv + kvh) << log_units) + (u & ((1 << log_units) - 1)) : 0;
    w.at = (uint64_t)a.k_pool + (uint64_t)slab * (kBlockTokens * kD * kElem);
    w.gone = __ballot(!mapped);
    w.scales = 0;
    if constexpr (kFormat == kBlkPools) {
      if (mapped) {
        const int64_t at = (int64_t)id * scale_row_bytes(a.Hkv) + kvh;
        w.scales = a.k_scales[at] | a.v_scales[at] << 8;
      }
    }
    return w;
  };
  int window_at = from / kWindowTiles * kWindowTiles;
  Window now = describe(window_at), then = describe(window_at + kWindowTiles);

  auto piece_of = [&](int i) __attribute__((always_inline)) { return ((kAlone ? 0 : wave * kLoads) + i) * 64 + this_lane(); };   // of a tile
  // kDirect: the memory unit writes 64 pieces in a row to LDS, so that each lane asks for the piece whose place is its own.
  const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  // The unit's bytes for that, of load 0: the others' differ by constants, and in bits that a constant turns over.
  const int first = piece_of(0) % kOfUnit / kPerToken, here = piece_of(0) % kPerToken;
  const int k_from = first * (kD * kElem) + k_place<kD>(first, here) % (kD * 2);
  const int v_from = first * (kD * kElem) + v_place<kD>(first, here) % (kD * 2);
  // A tile on its way: out of memory into registers, from there into LDS.
  u32x4 kr[kLoads], vr[kLoads];
  float ks[kOwn], vs[kOwn];   // of the units that it is from
#pragma unroll
  for (int x = 0; x < kOwn; ++x) ks[x] = vs[x] = 1.f;
  uint32_t unmapped = 0;      // of the tile that was asked for last, a bit for each unit that is not there
  auto ask = [&](int tile, int at_place) {
    if (tile >= window_at + kWindowTiles) {
      now = then;
      window_at += kWindowTiles;
      then = describe(window_at + kWindowTiles);
    }
    const int u0 = kUnits * (tile - window_at);
    unmapped = (uint32_t)(now.gone >> u0) & ((1 << kUnits) - 1);
#pragma unroll
    for (int x = 0; x < kOwn; ++x) {
      const int u = u0 + (kAlone ? x : wave * kLoads * 64 / kOfUnit);
      const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(now.at >> 32), u) << 32 |
                          (uint32_t)__builtin_amdgcn_readlane((int)now.at, u);
      const int rows = now.gone >> u & 1 ? 0 : min(kBlockTokens, context - (kUnits * window_at + u) * kBlockTokens), bytes = rows * (kD * kElem);
      const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, bytes, kRawBuffer);
      const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc((void*)(at + v_behind), 0, bytes, kRawBuffer);
      if constexpr (kFormat == kBlkPools) {
        const int both = __builtin_amdgcn_readlane(now.scales, u);
        ks[x] = __uint_as_float((uint32_t)(both & 0xff) << 23);
        vs[x] = __uint_as_float((uint32_t)(both >> 8) << 23);
      }
      int k0 = k_from, v0 = v_from;
      again(k0);
      again(v0);
      auto loads = [&](auto kind) __attribute__((always_inline)) {
        constexpr bool once = decltype(kind)::value;
#pragma unroll
        for (int y = 0; y < kEach; ++y) {
          const int i = x * kEach + y;
          if constexpr (kDirect) {
            constexpr int kTokens = 64 / kPerToken;   // of a load
            const uint32_t to_lds = lds_at + 2 * at_place * kTileBytes + 16 * 64 * ((kAlone ? 0 : wave * kLoads) + i);
            load_to_lds(kb, to_lds, (k0 ^ k_place<kD>(kTokens * y, 0) % (kD * 2)) + kTokens * y * kD * kElem, once);
            load_to_lds(vb, to_lds + kTileBytes, (v0 ^ v_place<kD>(kTokens * y, 0) % (kD * 2)) + kTokens * y * kD * kElem, once);
          } else if constexpr (kStaged) {
            const uint32_t to_lds = lds_at + 2 * kTileBytes + 16 * 64 * (wave * kLoads + i);
            const int offset = 16 * (piece_of(i) % kOfUnit);
            load_to_lds(kb, to_lds, offset, false);
            load_to_lds(vb, to_lds + 16 * kSource, offset, false);
          } else {
            const int offset = 16 * (piece_of(i) % kOfUnit);
            kr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kb, offset, 0, once ? 2 : 0));
            vr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vb, offset, 0, once ? 2 : 0));
          }
        }
      };
      if (kAlone && tok.only) loads(std::true_type{});
      else loads(std::false_type{});
    }
  };
  // What is not finite in V of keys that some row may not see does not go through the matrix product, where a weight of zero does not silence it: it
  // is held back, and the rows that see its key become NaN there in the end.  An infinite one, too, which in tiles that all rows see is infinite or NaN as
  // the product has it, and all of a block with a scale of 2^120 or more, which appends do not choose.
  auto hold_back = [&](int i, int tile, int t, int p) {
    constexpr int kValues = 16 / kElem;
    bool bad = false;
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const uint32_t w = vr[i][z];
      if constexpr (kFormat == 0) bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
      else bad |= (w & 0x7fu) == 0x7fu || (w & 0x7f00u) == 0x7f00u || (w & 0x7f0000u) == 0x7f0000u || (w & 0x7f000000u) == 0x7f000000u;
    }
    const bool all = kFormat == kBlkPools && !(vs[i / kEach] < kTooLarge);
    if (!bad && !all) return;
    any_bad = 1;
#pragma unroll
    for (int e = 0; e < kValues; ++e) {
      const int shift = 8 * kElem * (e % (4 / kElem));
      const uint32_t mask = kFormat == 0 ? 0x7f80u : 0x7fu;
      if (all || ((vr[i][e * kElem / 4] >> shift) & mask) == mask) {
        atomicMin(&first_bad[kValues * p + e], kKeyTile * tile + t);
        vr[i][e * kElem / 4] &= ~((kFormat == 0 ? 0xffffu : 0xffu) << shift);
      }
    }
  };
  // kDirect: what has arrived is in place; of a tile that is looked at this lane's pieces of V are read back.
  auto arrived = [&](int tile, char* v_lds, bool look) {
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    if (!look) return;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = piece_of(i);
      u32x4* at = (u32x4*)(v_lds + 16 * piece);
      vr[i] = *at;
      const u32x4 was = vr[i];
      hold_back(i, tile, piece / kPerToken, v_place<kD>(piece / kPerToken, piece % kPerToken) % (kD * 2) / 16);
      if (vr[i].x != was.x || vr[i].y != was.y || vr[i].z != was.z || vr[i].w != was.w) *at = vr[i];
    }
  };
  auto put = [&](int tile, char* k_lds, char* v_lds, bool look) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = piece_of(i);
      const int t = piece / kPerToken, p = piece % kPerToken;
      const float k_by = ks[i / kEach], v_by = look && !(vs[i / kEach] < kTooLarge) ? 1.f : vs[i / kEach];   // held back, all of it
      if (look) hold_back(i, tile, t, p);
      if constexpr (kFormat == 0) {
        *(u32x4*)(k_lds + k_place<kD>(t, p)) = kr[i];
        *(u32x4*)(v_lds + v_place<kD>(t, p)) = vr[i];
      } else {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const u32x2 k0 = widen(kr[i][2 * z], k_by), k1 = widen(kr[i][2 * z + 1], k_by);
          *(u32x4*)(k_lds + k_place<kD>(t, 2 * p + z)) = u32x4{k0.x, k0.y, k1.x, k1.y};
          const u32x2 v0 = widen(vr[i][2 * z], v_by), v1 = widen(vr[i][2 * z + 1], v_by);
          *(u32x4*)(v_lds + v_place<kD>(t, 2 * p + z)) = u32x4{v0.x, v0.y, v1.x, v1.y};
        }
      }
    }
  };

  float m = kLeast, l = 0.f;   // of row n: the reference maximum in log2 units, this lane's part of the sum
  f32x16 o[kTiles];             // o[d][r]: row n, dim 32*d + 8*(r / 4) + 4*h + r % 4
#pragma unroll
  for (int d = 0; d < kTiles; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;

  // Where this lane reads in LDS: a tile's places differ from these by constants, and in bits that a constant turns over.
  int k_base = k_place<kD>(n, h), v_base;
  const int v_key = 4 * h + ((lane & 15) >> 2), v_dim = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);   // this lane's part of what 16 lanes transpose
  v_base = v_place<kD>(v_key, v_dim >> 3) + 2 * (v_dim & 7);
  // V's operand of keys 16*step .. +15, dims 32*d .. +31
  auto v_operand = [&](const char* v_lds, int base, int step, int d) -> u32x4 {
    typedef __attribute__((address_space(3))) s16x4* Place;
    const char* at = v_lds + (base ^ 64 * (d & 3)) + 256 * (d >> 2) + 16 * step * kD * 2;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)at);
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(at + 8 * kD * 2));
    const u32x2 xx = __builtin_bit_cast(u32x2, x), yy = __builtin_bit_cast(u32x2, y);
    return u32x4{xx.x, xx.y, yy.x, yy.y};
  };

  auto attend = [&](const char* k_lds, const char* v_lds, int tile, uint32_t gone) __attribute__((always_inline)) {
    int k_at = k_base, v_at = v_base;
    again(k_at);
    f32x16 s[kHalves];
#pragma unroll
    for (int b = 0; b < kHalves; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
    for (int jj = 0; jj < kSteps; ++jj)
#pragma unroll
      for (int b = 0; b < kHalves; ++b) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, *(const u32x4*)(k_lds + (k_at ^ 32 * (jj & 7)) + 256 * (jj >> 3) + 32 * b * kD * 2));
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[jj], s[b], 0, 0, 0);
      }
    // some reads ahead of the products, else each waits for its own
    __builtin_amdgcn_sched_group_barrier(kDsRead, kReadsAhead, 0);
#pragma unroll
    for (int i = 0; i < kHalves * kSteps - kReadsAhead; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMfma, kReadsAhead, 0);
    const int key0 = kKeyTile * tile;
    if (gone != 0 || key0 + kKeyTile - 1 > wave_from) {
      asm volatile("");   // a branch: most tiles have nothing to mask
      const int here = this_lane();
      const int last_key = row_of(here).last_key, h = here >> 5;
#pragma unroll
      for (int b = 0; b < kHalves; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * b + 8 * (r >> 2) + 4 * h + (r & 3);
          s[b][r] = key0 + key <= last_key && !((gone >> (2 * b + (r >> 3))) & 1) ? s[b][r] : kNegInf;
        }
    }
    float most = s[0][0];
#pragma unroll
    for (int i = 1; i + 1 < 16 * kHalves; i += 2) most = fmaxf(fmaxf(most, s[i >> 4][i & 15]), s[(i + 1) >> 4][(i + 1) & 15]);
    most = fmaxf(most, s[kHalves - 1][15]);
    if (__any(most * scale > m + kLazyLog2)) {
      most = fmaxf(most, __shfl_xor(most, 32)) * scale;
      const float raised = fmaxf(m, most);
      const float alpha = __builtin_amdgcn_exp2f(m - raised);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m = raised;
    }
    [[maybe_unused]] u32x4 p[2 * kHalves];   // weights of keys 16*step .. +15, the B operand
    float sum[kHalves] = {};
#pragma unroll
    for (int b = 0; b < kHalves; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], scale, -m));
        sum[b] += s[b][r];
      }
      if constexpr (!kTwo)
#pragma unroll
        for (int z = 0; z < 8; ++z) p[2 * b + (z >> 2)][z & 3] = pack_bf16(s[b][2 * z], s[b][2 * z + 1]);
    }
    again(v_at);
    l += kHalves == 2 ? sum[0] + sum[kHalves - 1] : sum[0];
#pragma unroll
    for (int step = 0; step < 2 * kHalves; ++step) {
      if constexpr (kTwo) {
        // here, not with the exponentials, and the products of what the rounding left behind those of all dims: no more registers than one number takes
        u32x4 high, low, v[kTiles];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const float x = s[step >> 1][8 * (step & 1) + 2 * z], y = s[step >> 1][8 * (step & 1) + 2 * z + 1];
          high[z] = pack_bf16(x, y);
          low[z] = pack_bf16(x - __uint_as_float(high[z] << 16), y - __uint_as_float(high[z] & 0xffff0000u));
        }
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
          v[d] = v_operand(v_lds, v_at, step, d);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[d]), __builtin_bit_cast(bf16x8, high), o[d], 0, 0, 0);
        }
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[d]), __builtin_bit_cast(bf16x8, low), o[d], 0, 0, 0);
      } else {
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_operand(v_lds, v_at, step, d)), __builtin_bit_cast(bf16x8, p[step]),
                                                         o[d], 0, 0, 0);
      }
    }
  };

  for (int d = threadIdx.x; d < kD; d += kThreads) first_bad[d] = INT32_MAX;
  if (threadIdx.x == 0) any_bad = 0;
  __syncthreads();
  if constexpr (kAlone) {
    // Every wavefront has all rows and every fourth tile, in LDS of its own: nobody waits for another before the end.
    char *k_lds = lds + 2 * wave * kTileBytes, *v_lds = k_lds + kTileBytes;
    const int first_tile = from + wave;
    if (first_tile < to) ask(first_tile, wave);
    for (int tile = first_tile; tile < to; tile += kWaves) {
      const uint32_t gone = unmapped;
      const bool look = kKeyTile * tile + kKeyTile - 1 > tok.at;
      if constexpr (kDirect) {
        arrived(tile, v_lds, look);
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        attend(k_lds, v_lds, tile, gone);
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // has read the tile
        if (tile + kWaves < to) ask(tile + kWaves, wave);
      } else {
        put(tile, k_lds, v_lds, look);
        if (tile + kWaves < to) ask(tile + kWaves, wave);
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        attend(k_lds, v_lds, tile, gone);
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
      }
    }
  } else {
  ask(from, 0);
  auto one = [&](int tile, auto at_place) __attribute__((always_inline)) {
    constexpr int kAt = decltype(at_place)::value;
    char *k_lds = lds + 2 * kAt * kTileBytes, *v_lds = k_lds + kTileBytes;
    const uint32_t gone = unmapped;
    const bool look = kKeyTile * tile + kKeyTile - 1 > tok.at;
    if constexpr (kDirect) {   // the next tile goes where all have read the one before
      arrived(tile, v_lds, look);
      __syncthreads();
      if (tile + 1 < to) ask(tile + 1, 1 - kAt);
    } else if constexpr (kStaged) {
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // a wavefront reads what it asked for itself
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        kr[i] = *(const u32x4*)(lds + 2 * kTileBytes + 16 * piece_of(i));
        vr[i] = *(const u32x4*)(lds + 2 * kTileBytes + 16 * kSource + 16 * piece_of(i));
      }
      __syncthreads();
      put(tile, lds, lds + kTileBytes, look);
      if (tile + 1 < to) ask(tile + 1, 0);
      __syncthreads();
    } else {
      put(tile, k_lds, v_lds, look);
      if (tile + 1 < to) ask(tile + 1, 0);
      __syncthreads();
    }
    if (!idle && kKeyTile * tile <= wave_to) attend(kStaged ? lds : k_lds, kStaged ? lds + kTileBytes : v_lds, tile, gone);
  };
  for (int tile = from; tile < to; tile += 2) {
    one(tile, std::integral_constant<int, 0>{});
    if (tile + 1 < to) one(tile + 1, std::integral_constant<int, 1>{});
  }
  }
  if (a.id_faults && refused && threadIdx.x == 0) atomicAdd(a.id_faults, refused);
  if constexpr (kAlone) {
    // The rows of four wavefronts into the first one's, where a lane finds its own numbers.
    l += __shfl_xor(l, 32);
    f32x4* mine = (f32x4*)(lds + 2 * wave * kTileBytes) + lane;
    static_assert(2 * kTileBytes >= kTiles * 16 * 64 * 4);
    if (wave > 0) {
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) mine[(4 * d + g) * 64] = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
      if (h == 0) {
        stats_of[wave][0][n] = m;
        stats_of[wave][1][n] = l;
      }
    }
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < kWaves; ++w) {
      const float other = stats_of[w][0][n], most = fmaxf(m, other);
      const float mine_by = __builtin_amdgcn_exp2f(m - most), other_by = __builtin_amdgcn_exp2f(other - most);
      const f32x4* its = (const f32x4*)(lds + 2 * w * kTileBytes) + lane;
      m = most;
      l = l * mine_by + stats_of[w][1][n] * other_by;
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 x = its[(4 * d + g) * 64];
#pragma unroll
          for (int z = 0; z < 4; ++z) o[d][4 * g + z] = o[d][4 * g + z] * mine_by + x[z] * other_by;
        }
    }
  }

  const int own = this_lane();
  const Row row = row_of(own);
  const int half = own >> 5;
  if (!row.live) return;
  if (__builtin_expect(any_bad, 0)) {
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (first_bad[32 * d + 8 * (r >> 2) + 4 * half + (r & 3)] <= row.last_key) o[d][r] = __builtin_nanf("");
  }
  const float total = kAlone ? l : l + __shfl_xor(l, 32);
  const int64_t q_row = (int64_t)row.of_call * kD;
  if (__builtin_expect(__any(total == 0.f), 0)) {   // these rows have seen nothing, or nothing that weighs anything
    const ScalarLoad ids = (ScalarLoad)(a.block_tables + (int64_t)tok.s * a.MAXB);
    int key = from * kKeyTile;                      // the first of a block that is there
    while (key < min(context, to * kKeyTile) && (unsigned)ids[key >> a.log_block] >= (unsigned)a.NB) key = ((key >> a.log_block) + 1) << a.log_block;
    if (key >= to * kKeyTile || key > row.last_key) m = kNegInf;
  }
  if (tiles <= a.piece) {
    const float inv = inverse(m, total, a.out_scale);
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(u32x2*)(a.out + q_row + 32 * d + 8 * g + 4 * half) =
            finish_row4(f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]}, inv);
  } else {
    float* part = a.parts + (int64_t)blockIdx.y * a.T * a.Hq * kD + q_row;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(part + 32 * d + 8 * g + 4 * half) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    if (half == 0) *(f32x2*)(a.stats + ((int64_t)blockIdx.y * a.T * a.Hq + row.of_call) * 2) = f32x2{m, total};
  }
}

// The rows of contexts that were cut, from their pieces: D / 4 lanes to a row.
template <int kD>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptLaunch a, int per, int keys) {
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
  const int tiles = (L - n + last + 1 + keys - 1) / keys;
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
        if (i + z >= count) ml[z] = kNoStats;
      fold(p, ml, x);
    }
    *(u32x2*)(a.out + row * kD + dim) = finish_row4(p.x, inverse(p.m, p.l, a.out_scale));
  }
}

template <int kD, int kFormat, int kKeyTile, bool kAlone>
void launch_tiles(const PromptLaunch& a, const PromptPlan& plan, hipStream_t stream) {
  const dim3 grid((unsigned)(plan.slots * a.Hkv), plan.pieces);
  hipLaunchKernelGGL((prompt_attn_kernel<kD, kFormat, kKeyTile, kAlone>), grid, dim3(kThreads), 0, stream, a, plan.tokens, (int)plan.slots,
                     65536u / a.G + 1);
}
template <int kD, int kFormat>
void launch(const PromptLaunch& a, const PromptPlan& plan, hipStream_t stream) {
  if (plan.alone) launch_tiles<kD, kFormat, 32, true>(a, plan, stream);
  else if (plan.pieces == 1) launch_tiles<kD, kFormat, prompt_keys(kD, false), false>(a, plan, stream);
  else launch_tiles<kD, kFormat, prompt_keys(kD, true), false>(a, plan, stream);
  if (plan.pieces == 1) return;
  const int heads = 256 / (kD / 4);
  hipLaunchKernelGGL((prompt_join_kernel<kD>), dim3(a.T, (a.Hq + heads - 1) / heads), dim3(256), 0, stream, a, plan.tokens,
                     plan.alone ? 32 : prompt_keys(kD, true));
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
  p.threads = kThreads;
  p.alone = T <= (int64_t)S * (32 / G);   // what a request has fits a wavefront, if they have alike
  p.tokens = (p.alone ? 32 : 32 * kWaves) / G;
  p.slots = T / p.tokens + S;
  // Few workgroups over long contexts: those are cut.  Into as many pieces as give the least time by this estimate, in us: workgroups in turns of as many
  // as run at once, a tile 2 us with D = 128, a start 3 tiles, and the pieces' rows written and read.  A call that fills the card twice is not cut
  // (eight prompts of D = 256 in pieces 245 us, whole 206), and no more workgroups are made than eight times fill it (drafts of 32 requests: with a stop at
  // two times 144 us, at eight 125).  With few rows memory is the bound: as many pieces as fill the card once, where contexts are as long as they may be;
  // a request has one group of rows there, of the slots that are kept for more.  Pieces of them, drafts of 8 requests, us: 1 89, 2 54, 4 50, 8 40, 16 45.
  //   The host knows the bound on the lengths, not the lengths: with a bound far above them pieces are long and fewer have work.  Drafts of 32 requests with
  // up to 7658 tokens by their own bound 116 us, by 32768 and more 140; 512 tokens behind 32000 380, by 65536 458, by 131072 and more 650.
  const int keys = p.alone ? 32 : prompt_keys(D, true);
  const int64_t tiles = ((int64_t)max_ctx + keys - 1) / keys, groups = (p.alone ? S : p.slots) * Hkv, at_once = 256 * prompt_groups(D, keys, p.alone);
  const double tile_us = p.alone ? 0.5 : prompt_groups(D, keys, false) * (double)D / 128 * keys / 64, join_us = (double)T * G * Hkv * (D + 2) * 8 / 5e6;
  double least = 0;
  p.pieces = 1;
  for (int64_t n = 1; n <= kMaxPieces && 4 * n <= tiles + 3 && (n == 1 || (groups < 2 * at_once && groups * n <= 8 * at_once)); ++n) {
    const int64_t piece = (tiles + n - 1) / n;
    const double us = (double)((groups * n + at_once - 1) / at_once) * (piece + 3) * tile_us + (n > 1 ? 5 + n * (join_us + (p.alone ? 0.3 : 0)) : 0);
    if (n == 1 || us < least) {
      least = us;
      p.piece = (int)piece;
      p.pieces = (int)((tiles + piece - 1) / piece);
    }
  }
  // The longest work first, else it ends alone: 24 pieces of 1..900 tokens behind 0..4096, 3 turns of the card, 254 -> 220 us, at D = 128 413 -> 383, in 5
  // turns ten prompts 202 -> 197.  Not where all run at once (8.7 -> 9.0) nor in many turns, where a request's groups in a row share its keys in the caches
  // (sixteen prompts, 7 turns, 303 -> 307, 40 of them, 18 turns, 720 -> 749).
  const int64_t places = 256 * prompt_groups(D, prompt_keys(D, false), false);
  p.ordered = !p.alone && p.pieces == 1 && S > 1 && S <= 64 && groups > places && groups <= 6 * places;
  if (p.pieces == 1) p.piece = max_ctx / (p.alone ? 32 : prompt_keys(D, false)) + 1;
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
