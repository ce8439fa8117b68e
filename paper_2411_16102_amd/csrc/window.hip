// Sliding-window attention with sinks over the paged cache, and the rotary positions and append before it.
//
// A row at position p sees token t of its sequence if t <= p and (t > p - W or t < S).  Of a context of any length that
// is at most the pages of the sinks and those of the window, so the work of a row is a list of pages: sink pages, then
// window pages, one behind the other.  Counted along that list both conditions keep their form: a token u of it is
// seen by a row at place a if u <= a and (u > a - W or u < S), where a is p less the tokens left out between the two
// parts.  (Where pages are left out, the sink pages lie wholly before every window of the unit.)
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
// rotary positions and append: a workgroup per row
// ------------------------------------------------------------------------------
// Pair (i, i + dh/2) of a query or key head is turned by the angle of its axis' position; values go to their slot of the
// transposed tile as they are.
__global__ __launch_bounds__(256) void rope_append_kernel(const RopeArgs a) {
  const int row = blockIdx.x, half = a.head_dim / 2, dh = a.head_dim;
  const uint16_t *src = a.qkv + row * a.qkv_stride;
  const int page = a.row_page[row], slot = a.row_slot[row];
  for (int i = threadIdx.x; i < (a.n_q_heads + a.n_kv_heads) * half; i += 256) {
    const int head = i / half, e = i % half;
    const int pos = a.positions[(size_t)a.axis_of_pair[e] * a.n_rows + row];
    const float c = a.cos[(size_t)pos * half + e], s = a.sin[(size_t)pos * half + e];
    const float lo = bf16_to_f32(src[head * dh + e]), hi = bf16_to_f32(src[head * dh + half + e]);
    const uint32_t two = pack_bf16x2(lo * c - hi * s, hi * c + lo * s);
    uint16_t *dst;
    if (head < a.n_q_heads) {
      dst = a.q + row * a.q_stride + head * dh;
    } else {
      if (page < 0) continue;
      dst = a.kv_pool + (((size_t)page * 2 * a.n_kv_heads + head - a.n_q_heads) * 16 + slot) * dh;
    }
    dst[e] = (uint16_t)two;
    dst[half + e] = (uint16_t)(two >> 16);
  }
  if (page < 0) return;
  for (int i = threadIdx.x; i < a.n_kv_heads * dh; i += 256)
    a.kv_pool[(((size_t)page * 2 + 1) * a.n_kv_heads * dh + i) * 16 + slot] = src[(a.n_q_heads + a.n_kv_heads) * dh + i];
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
  if (a.n_rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(rope_append_kernel, dim3(a.n_rows), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace bs
