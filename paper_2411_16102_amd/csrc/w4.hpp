// Products of few rows with 4-bit weights (see blendstep_stream.h).
//
// The laid-out weight: blocks of 16 outputs by 128 inputs, all inputs of 16 outputs one behind the other; places past n
// and k hold zeros.  A block is 1 KB, 16 bytes for each of 64 lanes: lane (j = lane % 16, g = lane / 16) holds,
// in 32-bit word s, inputs 32 s + 8 g .. + 7 of output j, the operand of one 16x16x32 matrix instruction.  Within a word the
// even inputs stand in the low 16 bits, the odd ones in the high 16 (nibble i: input 2 i, nibble i + 4: input
// 2 i + 1), so that shifting and masking yields pairs of neighbours.  Behind the blocks come the scales, for each block [16 outputs][groups of
// 128 inputs] bf16, so that a lane has those of its output in one load, and, where there are any, the zero points in the same order, a byte each.
#pragma once
#include <stdint.h>
#include <hip/hip_runtime.h>

namespace bs {

struct W4Layout {
  int64_t n_blocks, k_blocks, groups;  // blocks of 16 outputs, of 128 inputs; groups of a padded row
  int64_t scales, zeros, bytes;        // offsets in bytes, and the whole
};
inline W4Layout w4_layout(int64_t n, int64_t k, int group, bool with_zeros) {
  W4Layout l;
  l.n_blocks = (n + 15) / 16;
  l.k_blocks = (k + 127) / 128;
  l.groups = l.k_blocks * (128 / group);
  l.scales = l.n_blocks * l.k_blocks * 1024;
  l.zeros = l.scales + l.n_blocks * l.groups * 32;
  l.bytes = l.zeros + (with_zeros ? l.n_blocks * l.groups * 16 : 0);
  return l;
}

struct W4Args {
  const uint16_t *x;
  const unsigned char *weight;
  uint16_t *y;
  int64_t x_stride, y_stride;
  int m, n, k, group;
  bool with_zeros;
  // partial sums of workgroups that share outputs, and their arrival counters (zero between launches)
  float *ws;
  unsigned *counters;
  size_t ws_floats;
  int n_counters, n_cu;
};
hipError_t launch_w4_linear(const W4Args &a, hipStream_t stream);
hipError_t launch_w4_pack(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, int64_t n, int64_t k, int group,
                          unsigned char *weight, hipStream_t stream);

}  // namespace bs
