// Launches of the stream pass over e4m3 pools with a scale for each block and KV head.
//
// The conversion of e4m3 to bf16 takes a scale in the same instruction, a power of two, so that scales cost no arithmetic and no rounding, only to know
// them: a lane loads both bytes of its unit's block when it describes the unit, 64 units at a time and ahead of their use, and the wavefront reads them
// from the lane after the next unit's loads have gone out.  Bound by memory as over pools with one scale: 64 requests of 1024..8192 tokens on 40/8 heads
// 97.7 us (6.0 TB/s) and with one scale 96.9; 32 long ones at D = 64 108.0 and 107.2; 4 short ones 6.6 and 6.8.
#include "attn_stream.h"

namespace pkv {
namespace {

template <int kD, typename Layer, bool kLarge>
void launch(const AttnLaunch& a, const BlockScales& scales, dim3 grid, size_t lds, hipStream_t stream) {
  Layer layer = {};
  static_cast<BlockScales&>(layer) = scales;
  hipLaunchKernelGGL((attn_stream_kernel<kD, true, Layer, kLarge>), grid, dim3(group_waves(kD) * 64), lds, stream, a, layer);
}

}  // namespace

hipError_t launch_attn_blk(const AttnLaunch& a_in, const uint8_t* k_scales, const uint8_t* v_scales, hipStream_t stream) {
  AttnLaunch a = a_in;
  const BlockScales scales = {k_scales, v_scales};
  const StreamLds l = stream_lds(a.S, a.G, a.D, true);
  a.staged_max = l.staged_max;
  a.wave_lds_floats = l.wave;
  a.turns = l.turn_bytes > 0;
  size_t lds = l.bytes + l.turn_bytes;
  if (!a.leaves_records) {
    // two records for each wavefront: nothing else is staged there
    a.wave_lds_floats = 2 * record_floats(a.G, a.D);
    a.staged_max = 1;
    lds = (l.prefix + group_waves(a.D) * a.wave_lds_floats) * sizeof(float) + l.turn_bytes;
    const dim3 grid(a.Hkv, 1, a.S);
    if (a.D == 64) launch<64, WholeBlkLayer, false>(a, scales, grid, lds, stream);
    else if (a.D == 128) launch<128, WholeBlkLayer, false>(a, scales, grid, lds, stream);
    else if (a.D == 256) launch<256, WholeBlkLayer, false>(a, scales, grid, lds, stream);
    else return hipErrorInvalidValue;
    return hipGetLastError();
  }
  const dim3 grid(a.waves / group_waves(a.D));
  if (a.D == 64) launch<64, BlkLayer, false>(a, scales, grid, lds, stream);
  else if (a.D == 128) launch<128, BlkLayer, false>(a, scales, grid, lds, stream);
  else if (a.D == 256) large_at_256(a) ? launch<256, BlkLayer, true>(a, scales, grid, lds, stream) : launch<256, BlkLayer, false>(a, scales, grid, lds, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
