// Device code of the rotary positions, shared by the appends to caches of either kind.
#pragma once
#include "attn_device.hpp"
#include "common.hpp"
#include "window.hpp"

namespace bs {
namespace rope_dev {
using namespace attn_dev;

constexpr int ROPE_THREADS = 256;

// cosines and sines of pairs e .. e + 7 (e a multiple of 8) at a row's positions
template <int DH, bool WHOLE>
__device__ __forceinline__ void angles_of(const RopeArgs &a, int row, int e, float (&c)[8], float (&s)[8]) {
  constexpr int HALF = DH / 2;
  if constexpr (WHOLE) {
    const size_t at = (size_t)a.positions[(size_t)a.axis_of_pair[e] * a.n_rows + row] * HALF + e;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4_t cv = *reinterpret_cast<const f32x4_t *>(a.cos + at + i), sv = *reinterpret_cast<const f32x4_t *>(a.sin + at + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        c[i + k] = cv[k];
        s[i + k] = sv[k];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const size_t at = (size_t)a.positions[(size_t)a.axis_of_pair[e + i] * a.n_rows + row] * HALF + e + i;
      c[i] = a.cos[at];
      s[i] = a.sin[at];
    }
  }
}

// query and key heads [h0, h1) of an item's rows; keys to their page
template <int DH, bool WHOLE>
__device__ __forceinline__ void turn_heads(const RopeArgs &a, const RopeItem &it, int h0, int h1) {
  constexpr int L = DH / 16, HALF = DH / 2;  // threads of a head
  const int t = threadIdx.x, e = t % L * 8;
  const int shift = it.n_rows > 8 ? 4 : it.n_rows > 4 ? 3 : it.n_rows > 2 ? 2 : it.n_rows > 1 ? 1 : 0;  // rows side by side: 2^shift
  const int r = (t / L) & ((1 << shift) - 1), step = (ROPE_THREADS / L) >> shift;
  if (r >= it.n_rows) return;
  const int row = it.row0 + r;
  float c[8], s[8];
  angles_of<DH, WHOLE>(a, row, e, c, s);
  const uint16_t *src = a.qkv + row * a.qkv_stride + e;
  uint16_t *to_q = a.q + row * a.q_stride + e;
  uint16_t *to_k = a.kv_pool + ((size_t)it.page * 2 * a.n_kv_heads * 16 + it.slot0 + r) * DH + e;
  auto turn = [&](int head, u32x4_t lo, u32x4_t hi) __attribute__((always_inline)) {
    u32x4_t lo2, hi2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float l0 = __uint_as_float(lo[i] << 16), l1 = __uint_as_float(lo[i] & 0xFFFF0000u);
      const float g0 = __uint_as_float(hi[i] << 16), g1 = __uint_as_float(hi[i] & 0xFFFF0000u);
      lo2[i] = pack_bf16x2(l0 * c[2 * i] - g0 * s[2 * i], l1 * c[2 * i + 1] - g1 * s[2 * i + 1]);
      hi2[i] = pack_bf16x2(g0 * c[2 * i] + l0 * s[2 * i], g1 * c[2 * i + 1] + l1 * s[2 * i + 1]);
    }
    if (head >= a.n_q_heads && it.page < 0) return;
    uint16_t *dst = head < a.n_q_heads ? to_q + head * DH : to_k + (size_t)(head - a.n_q_heads) * 16 * DH;
    *reinterpret_cast<u32x4_t *>(dst) = lo2;
    *reinterpret_cast<u32x4_t *>(dst + HALF) = hi2;
  };
  constexpr int U = 4;  // heads on the way
  int h = h0 + ((t / L) >> shift);
  for (; h + (U - 1) * step < h1; h += U * step) {
    u32x4_t lo[U], hi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      lo[u] = ld16(src + (h + u * step) * DH);
      hi[u] = ld16(src + (h + u * step) * DH + HALF);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) turn(h + u * step, lo[u], hi[u]);
  }
  for (; h < h1; h += step) turn(h, ld16(src + h * DH), ld16(src + h * DH + HALF));
}

}  // namespace rope_dev
}  // namespace bs
