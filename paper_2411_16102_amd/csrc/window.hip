// Sliding-window attention with sinks over the paged cache, and the rotary positions and append before it.
//
// A row at position p sees token t of its sequence if t <= p and (t > p - W or t < S).  Of a context of any length that
// is at most the pages of the sinks and those of the window, so the work of a row is a list of pages: sink pages, then
// window pages, one behind the other.  Counted along that list both conditions keep their form: a token u of it is
// seen by a row at place a if u <= a and (u > a - W or u < S), where a is p less the tokens left out between the two
// parts.  (Where pages are left out, the sink pages lie wholly before every window of the unit.)
#include <algorithm>

#include "attn_device.hpp"
#include "common.hpp"
#include "rope_device.hpp"
#include "window.hpp"
#include "window_device.hpp"

namespace bs {
namespace {
using namespace attn_dev;
using namespace window_dev;
using namespace rope_dev;

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void window_unit_kernel(const WindowArgs a) {
  __shared__ __align__(16) unsigned char lds[WINDOW_UNIT_LDS(DH, NW)];
  window_unit<DH, NW>(a, blockIdx.x, lds);
}

// ------------------------------------------------------------------------------
// rotary positions and append: a workgroup per run of rows in one page and share of the heads
// ------------------------------------------------------------------------------
// Pair (i, i + dh/2) of a query or key head is turned by the angle of its axis' position.  A thread holds eight pairs of one row
// (16 bytes of either half of a head) and the sines and cosines of their positions, for all of the heads that it takes.  Values go to
// slots of a transposed tile: more than four rows of a page are turned round in LDS, so that a thread stores eight slots of a
// dimension (16 bytes, where all eight are this step's); a few rows are stored from where they were read, 2 bytes a slot.
// Products and sums in 32 bits, one rounding.  Bound by moving the rows: 8 segments of a 64 + 8 head layer, 587 MB, 119 to 128 us, 4.6 to
// 4.9 TB/s (a large copy 4.9); axes in turn, a load for every angle, 12 % more; 77 single rows 4.1 us, a launch and two round trips.
template <int DH>
__device__ __forceinline__ void append_values(const RopeArgs &a, const RopeItem &it, int h0, int h1, uint16_t (*turned)[16][DH + 8]) {
  constexpr int L = DH / 8, PASS = ROPE_THREADS / (2 * DH);  // threads of a row of a head; heads that a pass takes
  static_assert(PASS * 2 * DH == ROPE_THREADS, "two threads per dimension");
  if (it.page < 0) return;  // the workgroup's
  const uint16_t *src = a.qkv + it.row0 * a.qkv_stride + (size_t)(a.n_q_heads + a.n_kv_heads) * DH;
  uint16_t *tile0 = a.kv_pool + ((size_t)it.page * 2 + 1) * a.n_kv_heads * 16 * DH;
  if (it.n_rows <= 4) {
    const int pieces = it.n_rows * (h1 - h0) * L;
    for (int i = threadIdx.x; i < pieces; i += ROPE_THREADS) {
      const int r = i / ((h1 - h0) * L), p = i % ((h1 - h0) * L), head = h0 + p / L, e = p % L * 8;
      const u32x4_t v = ld16(src + r * a.qkv_stride + head * DH + e);
      uint16_t *dst = tile0 + ((size_t)head * DH + e) * 16 + it.slot0 + r;
#pragma unroll
      for (int k = 0; k < 8; ++k) dst[16 * k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
    }
    return;
  }
  const int t = threadIdx.x;
  for (int head = h0; head < h1; head += PASS) {
    const int n = min(PASS, h1 - head);
#pragma unroll
    for (int k = 0; k < 16 * L * PASS / ROPE_THREADS; ++k) {
      const int i = k * ROPE_THREADS + t, e = i % L * 8, r = i / L % 16, h = i / (16 * L);
      if (h < n && r < it.n_rows) *reinterpret_cast<u32x4_t *>(&turned[h][it.slot0 + r][e]) = ld16(src + r * a.qkv_stride + (head + h) * DH + e);
    }
    __syncthreads();
    const int h = t / (2 * DH), d = t / 2 % DH, s0 = 8 * (t & 1);
    if (h < n) {
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = turned[h][s0 + k][d];
      uint16_t *dst = tile0 + ((size_t)(head + h) * DH + d) * 16 + s0;
      if (s0 >= it.slot0 && s0 + 8 <= it.slot0 + it.n_rows)
        *reinterpret_cast<u32x4_t *>(dst) = u32x4_t{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
      else
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (s0 + k >= it.slot0 && s0 + k < it.slot0 + it.n_rows) dst[k] = (uint16_t)v[k];
    }
    __syncthreads();
  }
}

template <int DH, bool WHOLE>
__global__ __launch_bounds__(ROPE_THREADS) void rope_append_kernel(const RopeArgs a, int shares, int v_shares) {
  __shared__ __align__(16) uint16_t turned[ROPE_THREADS / (2 * DH)][16][DH + 8];
  const int item = blockIdx.x / (shares + v_shares), share = blockIdx.x % (shares + v_shares);
  const RopeItem it = a.items[item];
  const int n = a.n_q_heads + a.n_kv_heads;
  if (share < shares) turn_heads<DH, WHOLE>(a, it, n * share / shares, n * (share + 1) / shares);
  else append_values<DH>(a, it, a.n_kv_heads * (share - shares) / v_shares, a.n_kv_heads * (share - shares + 1) / v_shares, turned);
}

}  // namespace

template <int DH>
static hipError_t launch_units(const WindowArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)a.n_items * (unsigned)a.s.n_kv_heads), block(64 * a.waves);
  if (a.waves == 1) hipLaunchKernelGGL((window_unit_kernel<DH, 1>), grid, block, 0, stream, a);
  else if (a.waves == 2) hipLaunchKernelGGL((window_unit_kernel<DH, 2>), grid, block, 0, stream, a);
  else if (a.waves == 4) hipLaunchKernelGGL((window_unit_kernel<DH, 4>), grid, block, 0, stream, a);
  else if (a.waves == 8) hipLaunchKernelGGL((window_unit_kernel<DH, 8>), grid, block, 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_window_units(const WindowArgs &a, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  if (a.s.head_dim == 128) return launch_units<128>(a, stream);
  if (a.s.head_dim == 64) return launch_units<64>(a, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_rope_append(const RopeArgs &a, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  // Shares of the heads: workgroups for a few rounds of the chip, of at least four heads
  const int heads = a.n_q_heads + a.n_kv_heads, rows = (a.n_rows + a.n_items - 1) / a.n_items;
  const int shares = std::max(1, std::min(2048 / a.n_items, heads / 4)), v_shares = rows > 4 ? a.n_kv_heads : 1;
  const dim3 grid((unsigned)a.n_items * (unsigned)(shares + v_shares)), block(ROPE_THREADS);
  if (a.head_dim == 128 && a.whole) hipLaunchKernelGGL((rope_append_kernel<128, true>), grid, block, 0, stream, a, shares, v_shares);
  else if (a.head_dim == 128) hipLaunchKernelGGL((rope_append_kernel<128, false>), grid, block, 0, stream, a, shares, v_shares);
  else if (a.head_dim == 64 && a.whole) hipLaunchKernelGGL((rope_append_kernel<64, true>), grid, block, 0, stream, a, shares, v_shares);
  else if (a.head_dim == 64) hipLaunchKernelGGL((rope_append_kernel<64, false>), grid, block, 0, stream, a, shares, v_shares);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace bs
