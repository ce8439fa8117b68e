// A paged cache in four bits: rotary positions and append, and conversions between its pages and bf16.
#include <algorithm>
#include <type_traits>

#include "../../include/blendstep_bits.h"
#include "common.hpp"
#include "context.hpp"
#include "kv4.hpp"
#include "kv4_device.hpp"
#include "rope_device.hpp"

namespace bs {
namespace {
using namespace attn_dev;
using namespace kv4_dev;
using namespace rope_dev;

// Codes of n_rows rows, in slots slot0 .. of one page, of KV heads [h0, h1).  A thread holds channels e .. e + 7 and those half a head further of
// a row's key or value; the dh / 16 threads of it find the least and greatest of each group by exchange.  A key's words are whole,
// a value's word has a code of each of eight tokens: codes meet in LDS, and words that the rows fill in part keep what they had.
// Arithmetic is 32 bits wide, without contraction.  source(kind, r, head): where a key (0) or value (1) begins; turn(lo, hi): its rotation.
template <int DH, int GROUP, class Source, class Turn>
__device__ __forceinline__ void append_codes(unsigned char *page, int n_rows, int slot0, int h0, int h1, unsigned char (*codes)[DH], Source &&source,
                                             Turn &&turn) {
  constexpr int L = DH / 16, HALF = DH / 2, R = GROUP >= HALF ? L : L / 2;  // R: threads that share a group
  constexpr int V = ROPE_THREADS / (2 * L);                                                 // rows of heads that a pass takes
  const int t = threadIdx.x, l = t % L, e = 8 * l, kind = t / L & 1, v = t / (2 * L);
  const int shift = n_rows > 8 ? 4 : n_rows > 4 ? 3 : n_rows > 2 ? 2 : n_rows > 1 ? 1 : 0;  // rows side by side: 2^shift
  const int r = v & ((1 << shift) - 1), slot = slot0 + r, heads = V >> shift;
  for (int h = h0; h < h1; h += heads) {
    const int head = h + (v >> shift);
    const bool ok = r < n_rows && head < h1;
    float x[2][8];
    {
      const uint16_t *src = source(kind, ok ? r : 0, ok ? head : h0) + e;
      const u32x4_t lo = ld16(src), hi = ld16(src + HALF);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[0][i] = __uint_as_float(i & 1 ? lo[i >> 1] & 0xFFFF0000u : lo[i >> 1] << 16);
        x[1][i] = __uint_as_float(i & 1 ? hi[i >> 1] & 0xFFFF0000u : hi[i >> 1] << 16);
      }
    }
    if (kind == 0) turn(r, x);
    float lo[2], hi[2];
    uint32_t far[2];  // the greatest magnitude's bits, which tell NaN and infinities
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      lo[k] = hi[k] = x[k][0];
      far[k] = __float_as_uint(x[k][0]) & 0x7FFFFFFFu;
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        lo[k] = fminf(lo[k], x[k][i]);
        hi[k] = fmaxf(hi[k], x[k][i]);
        far[k] = max(far[k], __float_as_uint(x[k][i]) & 0x7FFFFFFFu);
      }
    }
    if constexpr (GROUP == DH) {
      lo[0] = lo[1] = fminf(lo[0], lo[1]);
      hi[0] = hi[1] = fmaxf(hi[0], hi[1]);
      far[0] = far[1] = max(far[0], far[1]);
    }
#pragma unroll
    for (int k = 0; k < (GROUP == DH ? 1 : 2); ++k) {
#pragma unroll
      for (int o = 1; o < R; o <<= 1) {
        lo[k] = fminf(lo[k], __shfl_xor(lo[k], o, 64));
        hi[k] = fmaxf(hi[k], __shfl_xor(hi[k], o, 64));
        far[k] = max(far[k], (uint32_t)__shfl_xor((int)far[k], o, 64));
      }
    }
    unsigned char *block = page + (size_t)head * kv4_head_bytes(DH, GROUP);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = GROUP == DH ? 0 : k;
      const Numbers n = numbers_of(lo[j], hi[j], far[j] >= 0x7F800000u);
      uint32_t c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = code_for(n, x[k][i]);
      if (kind == 1) {
        const u32x2_t w = {c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24};
        *reinterpret_cast<u32x2_t *>(&codes[v][k * HALF + e]) = w;
      } else if (ok) {
        reinterpret_cast<uint32_t *>(block)[kv4_keys_at(l & 3, 4 * (slot >> 3) + (slot & 3), slot >> 2 & 1, (k * HALF + e) >> 5, DH)] = word_of(c);
      }
      if (ok && l % R == 0 && (GROUP < DH || k == 0)) {
        const int g = (k * HALF + e) / GROUP;
        *reinterpret_cast<uint16_t *>(block + kv4_number_at(slot, 2 * kind, g, DH, GROUP)) = (uint16_t)scale_bits(n);
        *reinterpret_cast<uint16_t *>(block + kv4_number_at(slot, 2 * kind + 1, g, DH, GROUP)) = (uint16_t)mid_bits(n);
      }
    }
    __syncthreads();
    // words of the halves of the page that have rows, a few of a thread on the way at a time
    const int half0 = slot0 >> 3, halves = ((slot0 + n_rows - 1) >> 3) - half0 + 1, n_words = min(heads, h1 - h) * halves * DH;
    constexpr int U = 4;
    for (int i0 = t; i0 < n_words; i0 += U * ROPE_THREADS) {
      uint32_t *at[U], old[U];
      int half[U], channel[U], ho[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min(i0 + u * ROPE_THREADS, n_words - 1), w = i % DH;
        const int rest = i / DH;
        half[u] = half0 + (halves == 2 ? rest & 1 : 0);
        ho[u] = halves == 2 ? rest >> 1 : rest;
        channel[u] = w / 64 * 64 + 16 * (w % 4) + w / 4 % 16;
        at[u] = reinterpret_cast<uint32_t *>(page + (size_t)(h + ho[u]) * kv4_head_bytes(DH, GROUP)) + kv4_values_at(half[u], channel[u], DH);
        old[u] = slot0 <= 8 * half[u] && slot0 + n_rows >= 8 * half[u] + 8 ? 0u : *at[u];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u * ROPE_THREADS >= n_words) break;
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int s = 8 * half[u] + j - slot0;
          c[j] = s >= 0 && s < n_rows ? codes[(ho[u] << shift) + s][channel[u]] : code_of(old[u], j);
        }
        *at[u] = word_of(c);
      }
    }
    __syncthreads();
  }
}

template <int DH, int GROUP, bool WHOLE>
__global__ __launch_bounds__(ROPE_THREADS) void rope_append4_kernel(const RopeArgs a, int shares, int kv_shares) {
  __shared__ __align__(16) unsigned char codes[ROPE_THREADS * 8 / DH][DH];
  const int item = blockIdx.x / (shares + kv_shares), share = blockIdx.x % (shares + kv_shares);
  const RopeItem it = a.items[item];
  if (share < shares) {
    turn_heads<DH, WHOLE>(a, it, a.n_q_heads * share / shares, a.n_q_heads * (share + 1) / shares);
    return;
  }
  if (it.page < 0) return;  // the workgroup's
  const int hkv = a.n_kv_heads, h0 = hkv * (share - shares) / kv_shares, h1 = hkv * (share - shares + 1) / kv_shares;
  unsigned char *page = reinterpret_cast<unsigned char *>(a.kv_pool) + (size_t)it.page * hkv * kv4_head_bytes(DH, GROUP);
  append_codes<DH, GROUP>(
      page, it.n_rows, it.slot0, h0, h1, codes,
      [&](int kind, int r, int head) { return a.qkv + (it.row0 + r) * a.qkv_stride + (size_t)(a.n_q_heads + kind * hkv + head) * DH; },
      [&](int r, float (&x)[2][8]) {
#pragma clang fp contract(off)
        float c[8], s[8];
        angles_of<DH, WHOLE>(a, it.row0 + min(r, it.n_rows - 1), threadIdx.x % (DH / 16) * 8, c, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float lo = x[0][i], hi = x[1][i];
          x[0][i] = lo * c[i] - hi * s[i];
          x[1][i] = hi * c[i] + lo * s[i];
        }
      });
}

template <int DH, int GROUP>
__global__ __launch_bounds__(ROPE_THREADS) void kv4_pack_kernel(const Kv4Pages p) {
  __shared__ __align__(16) unsigned char codes[ROPE_THREADS * 8 / DH][DH];
  const int64_t page = blockIdx.x / p.n_kv_heads;
  const int head = blockIdx.x % p.n_kv_heads;
  append_codes<DH, GROUP>(
      p.pool + (size_t)page * p.n_kv_heads * kv4_head_bytes(DH, GROUP), 16, 0, head, head + 1, codes,
      [&](int kind, int r, int h) { return (kind ? p.v_in : p.k_in) + ((page * 16 + r) * p.n_kv_heads + h) * DH; }, [](int, float (&)[2][8]) {});
}

// A workgroup per page and head, its block in LDS; a thread gives eight channels of a token.
template <int DH, int GROUP>
__global__ __launch_bounds__(256) void kv4_unpack_kernel(const Kv4Pages p) {
  constexpr int BYTES = kv4_head_bytes(DH, GROUP), C = DH / 8;
  __shared__ __align__(16) unsigned char block[BYTES];
  const int64_t page = blockIdx.x / p.n_kv_heads;
  const int head = blockIdx.x % p.n_kv_heads;
  const u32x4_t *src = reinterpret_cast<const u32x4_t *>(p.pool + ((size_t)page * p.n_kv_heads + head) * BYTES);
  for (int i = threadIdx.x; i < BYTES / 16; i += 256) reinterpret_cast<u32x4_t *>(block)[i] = src[i];
  __syncthreads();
  const uint32_t *words = reinterpret_cast<const uint32_t *>(block);
  for (int i = threadIdx.x; i < 2 * 16 * C; i += 256) {
    const int kind = i / (16 * C), t = i / C % 16, e = i % C * 8;
    const float scale = bf16_to_f32(*reinterpret_cast<const uint16_t *>(block + kv4_number_at(t, 2 * kind, e / GROUP, DH, GROUP)));
    const float mid = bf16_to_f32(*reinterpret_cast<const uint16_t *>(block + kv4_number_at(t, 2 * kind + 1, e / GROUP, DH, GROUP)));
    u32x4_t out;
    const uint32_t key = words[kv4_keys_at(e / 8 & 3, 4 * (t >> 3) + (t & 3), t >> 2 & 1, e >> 5, DH)];
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = value_of(scale, mid, kind ? code_of(words[kv4_values_at(t >> 3, e + k, DH)], t & 7) : code_of(key, k));
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
    *reinterpret_cast<u32x4_t *>((kind ? p.v_out : p.k_out) + ((page * 16 + t) * p.n_kv_heads + head) * DH + e) = out;
  }
}

// calls f with the head size and group as constants
template <class F>
hipError_t with_shape(int head_dim, int group, F &&f) {
  typedef std::integral_constant<int, 32> G32;
  typedef std::integral_constant<int, 64> G64;
  typedef std::integral_constant<int, 128> G128;
  if (head_dim == 128 && group == 128) return f(G128{}, G128{});
  if (head_dim == 128 && group == 64) return f(G128{}, G64{});
  if (head_dim == 128 && group == 32) return f(G128{}, G32{});
  if (head_dim == 64 && group == 64) return f(G64{}, G64{});
  if (head_dim == 64 && group == 32) return f(G64{}, G32{});
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_rope_append4(const RopeArgs &a, int group, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  // Shares of the query heads: workgroups for a few rounds of the chip, of at least four heads.  Of the KV heads: as many as a pass takes of a whole
  // page's rows (of few rows it takes them all, but a workgroup that has several waits for one after the other where others have whole pages).  A step of single tokens alone pays
  // for it: of each of eight workgroups 16 threads code, 77 rows of 8 KV heads 7.9 us where the append of bf16 takes 5.2.
  const int shares = std::max(1, std::min(2048 / a.n_items, a.n_q_heads / 4)), kv_shares = std::max(1, a.n_kv_heads * a.head_dim / 128);
  const dim3 grid((unsigned)a.n_items * (unsigned)(shares + kv_shares)), block(ROPE_THREADS);
  return with_shape(a.head_dim, group, [&](auto dh, auto g) {
    if (a.whole) hipLaunchKernelGGL((rope_append4_kernel<dh(), g(), true>), grid, block, 0, stream, a, shares, kv_shares);
    else hipLaunchKernelGGL((rope_append4_kernel<dh(), g(), false>), grid, block, 0, stream, a, shares, kv_shares);
    return hipGetLastError();
  });
}

hipError_t launch_kv4_pack(const Kv4Pages &p, hipStream_t stream) {
  if (p.n_pages <= 0) return hipSuccess;
  return with_shape(p.head_dim, p.group, [&](auto dh, auto g) {
    hipLaunchKernelGGL((kv4_pack_kernel<dh(), g()>), dim3((unsigned)(p.n_pages * p.n_kv_heads)), dim3(ROPE_THREADS), 0, stream, p);
    return hipGetLastError();
  });
}

hipError_t launch_kv4_unpack(const Kv4Pages &p, hipStream_t stream) {
  if (p.n_pages <= 0) return hipSuccess;
  return with_shape(p.head_dim, p.group, [&](auto dh, auto g) {
    hipLaunchKernelGGL((kv4_unpack_kernel<dh(), g()>), dim3((unsigned)(p.n_pages * p.n_kv_heads)), dim3(256), 0, stream, p);
    return hipGetLastError();
  });
}

}  // namespace bs

using namespace bs;

namespace {

int convert(bs_ctx *c, const char *what, const void *k, const void *v, const void *pool, int64_t n_pages, int32_t group, Kv4Pages *p) {
  const CtxView view = ctx_view(c);
  if (view.device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
  const int hkv = view.cfg->n_kv_heads, dh = view.cfg->head_dim;
  if (!kv4_shape(dh, group)) return ctx_fail(c, BS_EINVAL, "%s: groups of %d channels of %d are not supported", what, group, dh);
  // (a launch has less than 2^32 threads)
  if (n_pages < 0 || n_pages > 0xffffff || n_pages * hkv > 0xffffff) return ctx_fail(c, BS_EINVAL, "%s: n_pages=%lld out of range", what, (long long)n_pages);
  if (n_pages > 0 && (!k || !v || !pool || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(pool)) & 15)))
    return ctx_fail(c, BS_EINVAL, "%s: a pointer is NULL or not 16-byte aligned", what);
  CTX_HIP_TRY(c, hipSetDevice(view.device));
  *p = Kv4Pages{};
  p->n_kv_heads = hkv;
  p->head_dim = dh;
  p->group = group;
  p->n_pages = n_pages;
  p->pool = (unsigned char *)const_cast<void *>(pool);
  return BS_OK;
}

}  // namespace

extern "C" {

int64_t bs_kv4_page_bytes(const bs_ctx *c, int32_t group) {
  if (!c) return 0;
  const bs_layer_cfg &g = *ctx_view(c).cfg;
  return kv4_shape(g.head_dim, group) ? (int64_t)g.n_kv_heads * kv4_head_bytes(g.head_dim, group) : 0;
}

int bs_kv4_pack(bs_ctx *c, const void *k, const void *v, void *kv_pool, int64_t n_pages, int32_t group, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    Kv4Pages p;
    if (const int rc = convert(c, "bs_kv4_pack", k, v, kv_pool, n_pages, group, &p)) return rc;
    p.k_in = (const uint16_t *)k;
    p.v_in = (const uint16_t *)v;
    CTX_HIP_TRY(c, launch_kv4_pack(p, (hipStream_t)stream));
    return BS_OK;
  });
}

int bs_kv4_unpack(bs_ctx *c, const void *kv_pool, void *k, void *v, int64_t n_pages, int32_t group, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    Kv4Pages p;
    if (const int rc = convert(c, "bs_kv4_unpack", k, v, kv_pool, n_pages, group, &p)) return rc;
    p.k_out = (uint16_t *)k;
    p.v_out = (uint16_t *)v;
    CTX_HIP_TRY(c, launch_kv4_unpack(p, (hipStream_t)stream));
    return BS_OK;
  });
}

}  // extern "C"
