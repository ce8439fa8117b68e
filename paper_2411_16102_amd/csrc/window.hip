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
#include "window.hpp"

namespace bs {
namespace {
using namespace attn_dev;

// Elements of a row that no row of the unit sees are never multiplied into a result: scores become -inf, values zero
// (a slot that was never written may hold NaN, and zero times NaN is NaN).
__device__ __forceinline__ uint32_t keep_two(uint32_t v, bool lo, bool hi) {
  return (lo ? v & 0x0000FFFFu : 0u) | (hi ? v & 0xFFFF0000u : 0u);
}

// ------------------------------------------------------------------------------
// narrow work: one wavefront per (item, KV head), its 16 columns are (row, head of the group)
// ------------------------------------------------------------------------------
// S^T = K Q^T and O^T = V^T P^T as in the decode units of the blended step: a lane owns one column, a pair of pages is
// one contraction of the second product, and the keys enter the first in the order that leaves a lane
// the probabilities of eight adjacent tokens of one page.
template <int DH>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2, 2))) void window_unit_kernel(const WindowArgs a) {
  constexpr int KC = DH / 32, DB = DH / 16;
  const int hkv = a.s.n_kv_heads, hq = a.s.n_q_heads, grp = hq / hkv;
  const int lane = threadIdx.x & 63, jq = lane & 15, g4 = lane >> 4;
  const WindowItem it = a.items[blockIdx.x / hkv];
  const int kvh = blockIdx.x % hkv;
  const size_t tile = (size_t)16 * DH;
  const float sc = a.s.scale_log2e;
  const bool ok = jq < it.n_rows * grp;
  const int row = it.row0 + (ok ? jq / grp : 0), head = kvh * grp + (ok ? jq % grp : 0);
  const int at = it.at + (ok ? jq / grp : 0);
  const int at_last = it.at + it.n_rows - 1;

  bf16x8_t qf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (ok) v = ld16(a.q + row * a.q_stride + head * DH + 32 * c + 8 * g4);
    qf[c] = as_bf16x8(v);
  }
  f32x4_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = NEG_BIG, l = 0.f;

  const int n_pg = it.n_pages;
  for (int pr = 0; 2 * pr < n_pg; ++pr) {
    const size_t p0 = a.item_pages[it.page_off + 2 * pr], p1 = a.item_pages[it.page_off + min(2 * pr + 1, n_pg - 1)];
    const uint16_t *b0 = a.kv_pool + (p0 * 2 * hkv + kvh) * tile, *b1 = a.kv_pool + (p1 * 2 * hkv + kvh) * tile;
    const uint16_t *kp = (jq < 8 ? b0 : b1) + (8 * ((jq >> 2) & 1) + (jq & 3)) * DH + 8 * g4;
    const uint16_t *vp = (g4 < 2 ? b0 : b1) + (size_t)hkv * tile + jq * 16 + 8 * (g4 & 1);
    u32x4_t k[2][KC], v[DB];
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      k[0][c] = ld16(kp + 32 * c);
      k[1][c] = ld16(kp + 4 * DH + 32 * c);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) v[db] = ld16(vp + db * 256);
    f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k[0][c]), qf[c], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k[1][c]), qf[c], s1, 0, 0, 0);
    }
    const int u0 = 32 * pr + 8 * g4;  // this lane's eight tokens
    float sv[8];
    bool any[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int u = u0 + r;
      sv[r] = r < 4 ? s0[r] : s1[r - 4];
      if (u > at || (u <= at - a.window && u >= it.sinks)) sv[r] = -INFINITY;
      any[r] = u <= at_last && (u > it.at - a.window || u < it.sinks) && u < 16 * n_pg;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int w = 0; w < 4; ++w) v[db][w] = keep_two(v[db][w], any[2 * w], any[2 * w + 1]);
    if (32 * pr + 16 >= 16 * n_pg) {  // the second page of the pair does not exist
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (g4 >= 2) sv[r] = -INFINITY;
    }
    float mx = sv[0];
#pragma unroll
    for (int r = 1; r < 8; ++r) mx = fmaxf(mx, sv[r]);
    mx *= sc;
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] *= alpha;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      sv[r] = fast_exp2(__builtin_fmaf(sv[r], sc, -m));
      l += sv[r];
    }
    const u32x4_t pw = {pack_bf16x2(sv[0], sv[1]), pack_bf16x2(sv[2], sv[3]), pack_bf16x2(sv[4], sv[5]), pack_bf16x2(sv[6], sv[7])};
#pragma unroll
    for (int db = 0; db < DB; ++db)
      o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v[db]), as_bf16x8(pw), o[db], 0, 0, 0);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (!ok) return;
  if (it.state >= 0) {
    const size_t base = (size_t)(it.state + jq / grp) * hq + head;
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4_t *>(a.part_acc + base * DH + 16 * db + 4 * g4) = o[db];
    if (g4 == 0) {
      a.part_m[base] = m;
      a.part_l[base] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing gives zeros; a NaN stays one)
  uint16_t *dst = a.out + row * a.out_stride + head * DH + 4 * g4;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    u32x2_t w;
    w.x = pack_bf16x2(o[db][0] * inv, o[db][1] * inv);
    w.y = pack_bf16x2(o[db][2] * inv, o[db][3] * inv);
    *reinterpret_cast<u32x2_t *>(dst + 16 * db) = w;
  }
}

// dh / 4 lanes per (row, head), four elements per lane: M = max m_p, out = sum 2^(m_p - M) acc_p / sum 2^(m_p - M) l_p
template <int DH>
__global__ __launch_bounds__(256) void window_join_kernel(const WindowArgs a) {
  constexpr int LPH = DH / 4;
  const int hq = a.s.n_q_heads;
  const long unit = ((long)blockIdx.x * 256 + threadIdx.x) / LPH;
  if (unit >= (long)a.n_joins * hq) return;
  const int32_t *j = a.joins + 4 * (unit / hq);
  const int head = (int)(unit % hq), li = threadIdx.x % LPH;
  float mx = NEG_BIG, ls = 0.f;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < j[3]; ++p) {
    const size_t at = (size_t)(j[1] + p * j[2]) * hq + head;
    const float m = a.part_m[at], m_new = fmaxf(mx, m), alpha = fast_exp2(mx - m_new), w = fast_exp2(m - m_new);
    mx = m_new;
    ls = ls * alpha + w * a.part_l[at];
    acc = acc * alpha + w * *reinterpret_cast<const f32x4_t *>(a.part_acc + at * DH + li * 4);
  }
  const float inv = ls == 0.f ? 0.f : 1.f / ls;
  u32x2_t o2;
  o2.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  o2.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2_t *>(a.out + j[0] * a.out_stride + head * DH + li * 4) = o2;
}

// ------------------------------------------------------------------------------
// rotary positions and append: a workgroup per run of rows in one page and share of the heads
// ------------------------------------------------------------------------------
// Pair (i, i + dh/2) of a query or key head is turned by the angle of its axis' position.  A thread holds eight pairs of one row
// (16 bytes of either half of a head) and the sines and cosines of their positions, for all of the heads that it takes.  Values go to
// slots of a transposed tile: more than four rows of a page are turned round in LDS, so that a thread stores eight slots of a
// dimension (16 bytes, where all eight are this step's); a few rows are stored from where they were read, 2 bytes a slot.
constexpr int ROPE_THREADS = 256;

template <int DH, bool WHOLE>
__device__ __forceinline__ void turn_heads(const RopeArgs &a, const RopeItem &it, int h0, int h1) {
  constexpr int L = DH / 16, HALF = DH / 2;  // threads of a head
  const int t = threadIdx.x, e = t % L * 8;
  const int shift = it.n_rows > 8 ? 4 : it.n_rows > 4 ? 3 : it.n_rows > 2 ? 2 : it.n_rows > 1 ? 1 : 0;  // rows side by side: 2^shift
  const int r = (t / L) & ((1 << shift) - 1), step = (ROPE_THREADS / L) >> shift;
  if (r >= it.n_rows) return;
  const int row = it.row0 + r;
  float c[8], s[8];
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

hipError_t launch_window_units(const WindowArgs &a, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)a.n_items * (unsigned)a.s.n_kv_heads);
  if (a.s.head_dim == 128) hipLaunchKernelGGL(window_unit_kernel<128>, grid, dim3(64), 0, stream, a);
  else if (a.s.head_dim == 64) hipLaunchKernelGGL(window_unit_kernel<64>, grid, dim3(64), 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_window_join(const WindowArgs &a, hipStream_t stream) {
  if (a.n_joins <= 0) return hipSuccess;
  const long threads = (long)a.n_joins * a.s.n_q_heads * (a.s.head_dim / 4);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (a.s.head_dim == 128) hipLaunchKernelGGL(window_join_kernel<128>, grid, dim3(256), 0, stream, a);
  else if (a.s.head_dim == 64) hipLaunchKernelGGL(window_join_kernel<64>, grid, dim3(256), 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
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
