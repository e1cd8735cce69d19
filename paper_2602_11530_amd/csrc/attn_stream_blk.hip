// Launches of the stream pass over e4m3 pools with a scale for each block and KV head.
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
