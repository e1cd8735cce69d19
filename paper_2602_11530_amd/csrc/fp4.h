// Pools held in 4 bits: E2M1 codes (a sign, two exponent bits with bias 1, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), and for each 32 dims
// of a token and KV head a scale byte b that stands for 2^(b - 127), 255 for NaN.
//
// The unit of a pool is a tile: 16 tokens of one KV head, codes and then scales, in the order in which the stream pass's lanes hold
// them, so that each of its loads is one row of bytes in a row:
//   K codes [D / 32][16 tokens][16 bytes]: a group of 32 dims
//   V codes [4][D / w][4 tokens][w / 2 bytes], w = 8 dims (4 at D = 64): token t is at [t / 4][.][t % 4]
//   scales  [D / 32][16 tokens]
// The lower half of a byte is the lower dim.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pkv {

__host__ __device__ constexpr int fp4_tile_bytes(int D) { return 8 * D + D / 2; }
// Byte of a tile where a token's eight dims 8 * chunk .. + 7 of K begin (four bytes), its dims `dim` .. + w - 1 of V, and a group's scale.
__host__ __device__ constexpr int fp4_k_place(int chunk, int token) { return 256 * (chunk >> 2) + 16 * token + 4 * (chunk & 3); }
__host__ __device__ constexpr int fp4_v_place(int D, int dim, int token) {
  return D == 64 ? 128 * (token >> 2) + 8 * (dim >> 2) + 2 * (token & 3) : 2 * D * (token >> 2) + 16 * (dim >> 3) + 4 * (token & 3);
}
__host__ __device__ constexpr int fp4_scale_place(int D, int group, int token) { return 8 * D + 16 * group + token; }

}  // namespace pkv
