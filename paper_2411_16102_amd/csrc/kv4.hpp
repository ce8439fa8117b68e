// A paged cache in four bits (see blendstep_bits.h): where things stand in a page, and the kernels that write and read it.
//
// A page holds, for each KV head, one block behind the other:
//   keys    words [2 i][4 g][8 r][4 s] (64-wide heads: [4 g][8 r][2 i][2 s]): codes of channels 32 s + 8 g .. + 7 of token 8 (r / 4) + 4 i + r % 4
//   values  words [dh / 64][2 halves][16][4 b]: codes of tokens 8 half .. + 7 of channel 64 first + 16 b + third index
//   numbers bf16  [2 halves][group][kind][8]: of tokens 8 half .. + 7; kinds: scale and mid of keys, then of values
// so that a lane of a matrix product's operand loads its part of a page 16 bytes at a time, neighbours side by side.  Element j of a word is at bits
// 4 (j / 2) + 16 (j % 2), turned left by 3: a shift, an and and an or make two bf16 numbers 16 + code of it (see kv4_device.hpp).
#pragma once
#include <stdint.h>
#include <hip/hip_runtime.h>
#include "window.hpp"

namespace bs {

// whether a cache of such heads and groups is supported
constexpr bool kv4_shape(int head_dim, int group) {
  return (head_dim == 64 || head_dim == 128) && (group == 32 || group == 64 || group == 128) && group <= head_dim;
}
constexpr int kv4_head_bytes(int head_dim, int group) { return 16 * head_dim + 128 * (head_dim / group); }
constexpr int kv4_keys_at(int g4, int r8, int i, int s, int head_dim) {  // word
  return head_dim == 128 ? ((i * 4 + g4) * 8 + r8) * 4 + s : ((g4 * 8 + r8) * 2 + i) * 2 + s;
}
constexpr int kv4_values_at(int half, int channel, int head_dim) {  // word
  return 2 * head_dim + ((channel / 64 * 2 + half) * 16 + channel % 16) * 4 + channel / 16 % 4;
}
constexpr int kv4_number_at(int token, int kind, int g, int head_dim, int group) {  // byte
  return 16 * head_dim + (token >> 3) * 64 * (head_dim / group) + (g * 4 + kind) * 16 + (token & 7) * 2;
}

// bs_rope_append into such a cache: the queries turned, keys turned and coded, values coded.
hipError_t launch_rope_append4(const RopeArgs &a, int group, hipStream_t stream);

struct Kv4Pages {
  int n_kv_heads, head_dim, group;
  int64_t n_pages;
  const uint16_t *k_in, *v_in;  // token-major [n_pages][16][Hkv][dh]
  uint16_t *k_out, *v_out;
  unsigned char *pool;
};
hipError_t launch_kv4_pack(const Kv4Pages &p, hipStream_t stream);
hipError_t launch_kv4_unpack(const Kv4Pages &p, hipStream_t stream);

// The narrow work of window attention over such a cache (a.kv_pool), and the wavefronts of it that the registers of a SIMD hold.
constexpr int kv4_resident(int head_dim, int group, int heads) { return head_dim == 128 ? (heads == 2 || group == 32 ? 2 : 3) : heads == 2 ? 3 : 4; }
hipError_t launch_window_units4(const WindowArgs &a, int group, hipStream_t stream);
// Rows of longer segments: items of up to KV4_ROW_BLOCKS blocks of sixteen columns for each of four wavefronts, with all of their pages.  Four groups to a head
// leave no registers for two blocks (62 spilled): at 1.3 to 2.7 times the time of narrow work from the largest to the smallest sizes, these stay narrow work.
constexpr int KV4_ROW_BLOCKS = 2;
inline bool kv4_has_rows(int head_dim, int group) { return head_dim / group <= 2; }
hipError_t launch_window_rows4(const WindowArgs &a, int group, hipStream_t stream);

}  // namespace bs
