// Device code of the narrow work of window attention, shared by the launches that run it.
#pragma once
#include "attn_device.hpp"
#include "common.hpp"
#include "join.hpp"
#include "window.hpp"

namespace bs {
namespace window_dev {
using namespace attn_dev;

// ------------------------------------------------------------------------------
// narrow work: a workgroup per (item, KV head); its 16 columns are (row, head of the group)
// ------------------------------------------------------------------------------
// S^T = K Q^T and O^T = V^T P^T as in the decode units of the blended step: a lane owns one column, a pair of pages is
// one contraction of the second product, and the keys enter the first in the order that leaves a lane
// the probabilities of eight adjacent tokens of one page.  Two sets of registers take the pairs in turn, one being
// computed while the other is on the way.  Elements that no row of the unit sees are never multiplied into a result: scores
// become -inf, values zero (a slot that was never written may hold NaN, and zero times NaN is NaN); pairs that all
// rows see whole, which is most of them, need neither.
//
// Probabilities are rounded to bf16 for their product with V (at most 2^-8 of the sum of p |v|, as elsewhere in this
// library); scores, statistics and accumulators are 32 bits wide.  Bound by reading the pages: 256 streams of window 1024, 8 KV
// heads (1.07 GB) take 175 us, 6.1 TB/s, what reads alone reach; 129 streams and two segments of a 64-wide layer (141 MB) 29 us, 4.9 TB/s; one
// stream 8.7 us: a launch, a round trip each for the plan, the pages and the join.
template <int DH>
struct Columns {  // the softmax of a wavefront's columns
  f32x4_t o[DH / 16];
  float m, l;
};

// pages [pg0, pg1) of the unit, at most 64
template <int DH>
__device__ __forceinline__ void walk_pages(const WindowArgs &a, const WindowItem &it, int kvh, int lane, int pg0, int pg1, const bf16x8_t (&qf)[DH / 32],
                                           Columns<DH> &c) {
  constexpr int KC = DH / 32, DB = DH / 16;
  const int hkv = a.s.n_kv_heads, grp = a.s.n_q_heads / hkv;
  const int jq = lane & 15, g4 = lane >> 4;
  const size_t tile = (size_t)16 * DH;
  const float sc = a.s.scale_log2e;
  const bool ok = jq < it.n_rows * grp;
  const int j = ok ? jq / grp : 0;
  // places are counted from this wavefront's first page
  const int n_pg = pg1 - pg0, first = it.at - 16 * pg0, last = first + it.n_rows - 1, at = first + j, sinks = it.sinks - 16 * pg0;
  const int my_page = a.item_pages[it.page_off + pg0 + min(lane, n_pg - 1)];  // lane i holds page i
  struct Frags {
    u32x4_t k[2][KC], v[DB];
  };
  const uint32_t k_off = (uint32_t)((8 * ((jq >> 2) & 1) + (jq & 3)) * DH + 8 * g4), v_off = (uint32_t)(jq * 16 + 8 * (g4 & 1));
  auto load = [&](int pr, Frags &f) __attribute__((always_inline)) {  // (past the end: the last page again, not used)
    const size_t p0 = (size_t)__builtin_amdgcn_readlane(my_page, min(2 * pr, n_pg - 1)), p1 = (size_t)__builtin_amdgcn_readlane(my_page, min(2 * pr + 1, n_pg - 1));
    const uint16_t *b0 = a.kv_pool + (p0 * 2 * hkv + kvh) * tile, *b1 = a.kv_pool + (p1 * 2 * hkv + kvh) * tile;
    const uint16_t *kp = (jq < 8 ? b0 : b1) + k_off, *vp = (g4 < 2 ? b0 : b1) + (size_t)hkv * tile + v_off;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      f.k[0][i] = ld16_kv<true>(kp + 32 * i);
      f.k[1][i] = ld16_kv<true>(kp + 4 * DH + 32 * i);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) f.v[db] = ld16_kv<true>(vp + db * 256);
  };
  auto compute = [&](int pr, Frags &f) __attribute__((always_inline)) {
    const int tb = 32 * pr;
    if (2 * pr >= n_pg) return;  // wave-uniform
    f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(f.k[0][i]), qf[i], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(f.k[1][i]), qf[i], s1, 0, 0, 0);
    }
    const int u0 = tb + 8 * g4;  // this lane's eight tokens
    float sv[8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sv[r] = s0[r];
      sv[4 + r] = s1[r];
    }
    const bool whole = tb + 32 <= 16 * n_pg && tb + 31 <= first && (tb > last - a.window || tb + 32 <= sinks);
    if (!whole) {  // wave-uniform
      const int end = min(16 * n_pg, last + 1);  // tokens from here on, and those of [sinks, unseen), are seen by no row
      const int unseen = first - a.window + 1;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        // (One condition, selected by: of an element that is written behind || and && the compiler made branches whose intermediate code is
        // right, and machine code that is not: -inf is written ahead of them, taken back for lanes that pass the first condition, and the block
        // for those that fail a later one is empty.)
        const int u = u0 + r;
        const bool hidden = (u > at) | ((u <= at - a.window) & (u >= sinks)) | (u >= 16 * n_pg);
        sv[r] = hidden ? -INFINITY : sv[r];
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) f.v[db] = mask_between8(mask_tokens8(f.v[db], u0, end), u0, sinks, unseen);
    }
    float mx = sc * fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
    if (__builtin_amdgcn_ballot_w64(mx > c.m + TAU) != 0) {  // (see TAU: the reference moves rarely)
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = fmaxf(c.m, mx), alpha = fast_exp2(c.m - m_new);
      c.m = m_new;
      c.l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) c.o[db] *= alpha;
    }
    float ps = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      sv[r] = fast_exp2(__builtin_fmaf(sv[r], sc, -c.m));
      ps += sv[r];
    }
    c.l += ps;
    const u32x4_t pw = {pack_bf16x2(sv[0], sv[1]), pack_bf16x2(sv[2], sv[3]), pack_bf16x2(sv[4], sv[5]), pack_bf16x2(sv[6], sv[7])};
#pragma unroll
    for (int db = 0; db < DB; ++db)
      c.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(f.v[db]), as_bf16x8(pw), c.o[db], 0, 0, 0);
  };
  Frags fa, fb;
  load(0, fa);
  load(1, fb);
  for (int pr = 0; 2 * pr < n_pg; pr += 2) {
    compute(pr, fa);
    load(pr + 2, fa);
    compute(pr + 1, fb);
    load(pr + 3, fb);
  }
}

// four results of a column (jq: its number among those of KV head kvh), dh = 16 db + 4 g4 ..
__device__ __forceinline__ void store_quad(const WindowArgs &a, const WindowItem &it, int kvh, int jq, int dh, int lane, int db, f32x4_t o, float l) {
  const int grp = a.s.n_q_heads / a.s.n_kv_heads;
  const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing gives zeros; a NaN stays one)
  u32x2_t w;
  w.x = pack_bf16x2(o[0] * inv, o[1] * inv);
  w.y = pack_bf16x2(o[2] * inv, o[3] * inv);
  *reinterpret_cast<u32x2_t *>(a.out + (it.row0 + jq / grp) * a.out_stride + (kvh * grp + jq % grp) * dh + 16 * db + 4 * (lane >> 4)) = w;
}

// LDS of a workgroup of NW wavefronts
constexpr int WINDOW_UNIT_LDS(int dh, int nw) { return (nw > 1 ? nw * (dh / 16) * 1024 : 0) + nw * 128 + 16; }

// The pages of a cache in bf16, as a unit walks them.
template <int DH>
struct Bf16Pages {
  __device__ __forceinline__ explicit Bf16Pages(const bf16x8_t (&)[DH / 32]) {}
  __device__ __forceinline__ void walk(const WindowArgs &a, const WindowItem &it, int kvh, int lane, int pg0, int pg1, const bf16x8_t (&qf)[DH / 32],
                                       Columns<DH> &c) {
    walk_pages<DH>(a, it, kvh, lane, pg0, pg1, qf, c);
  }
  __device__ __forceinline__ void finish(Columns<DH> &) {}
  static constexpr int HEADS = 1;  // KV heads whose columns share a wavefront
  static constexpr int joined(int blocks) { return blocks <= 4 ? 8 : 4; }  // states of so many blocks that a join has on the way
};

template <int DH, int NW, class Pages = Bf16Pages<DH>>
__device__ __forceinline__ void window_unit(const WindowArgs &a, int block, unsigned char *lds) {
  constexpr int DB = DH / 16;
  constexpr int CPH = 16 / Pages::HEADS;  // columns of a KV head
  const int grp = a.s.n_q_heads / a.s.n_kv_heads, hkv = a.s.n_kv_heads / Pages::HEADS, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WindowItem it = a.items[block / hkv];
  const int kvh = block % hkv;  // (times HEADS: the first of the KV heads)
  const int col = (lane & 15) % CPH, col_head = kvh * Pages::HEADS + (lane & 15) / CPH;
  const bool ok = col < it.n_rows * grp;
  // pairs of pages in nearly equal shares
  const int n_pairs = (it.n_pages + 1) >> 1;
  const int pg0 = 2 * (int)((int64_t)n_pairs * wave / NW), pg1 = min(it.n_pages, 2 * (int)((int64_t)n_pairs * (wave + 1) / NW));
  bf16x8_t qf[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) {
    const int jq = ok ? col : 0;
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (ok) v = ld16(a.q + (it.row0 + jq / grp) * a.q_stride + (col_head * grp + jq % grp) * DH + 32 * i + 8 * (lane >> 4));
    qf[i] = as_bf16x8(v);
  }
  Columns<DH> c;
#pragma unroll
  for (int db = 0; db < DB; ++db) c.o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  c.m = NEG_BIG;
  c.l = 0.f;
  Pages pages(qf);
  for (int pg = pg0; pg < pg1; pg += 64) pages.walk(a, it, kvh * Pages::HEADS, lane, pg, min(pg + 64, pg1), qf, c);
  pages.finish(c);
  c.l += __shfl_xor(c.l, 16, 64);
  c.l += __shfl_xor(c.l, 32, 64);
  if constexpr (NW == 1) {
    if (it.state < 0) {
      if (ok)
#pragma unroll
        for (int db = 0; db < DB; ++db) store_quad(a, it, col_head, col, DH, lane, db, c.o[db], c.l);
      return;
    }
  }
  // The workgroup's wavefronts meet in LDS: blocks of 16 dimensions are dealt among them.
  constexpr int MINE = NW < DB ? DB / NW : 1;  // blocks of a wavefront
  f32x4_t (*acc)[DB][64] = reinterpret_cast<f32x4_t (*)[DB][64]>(lds);
  float (*ml)[2][16] = reinterpret_cast<float (*)[2][16]>(lds + (NW > 1 ? NW * DB * 1024 : 0));
  unsigned *flag = reinterpret_cast<unsigned *>(lds + WINDOW_UNIT_LDS(DH, NW) - 16);
  f32x4_t o[MINE];
  float m = c.m, l = c.l;
  if constexpr (NW == 1) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) o[i] = c.o[i];
  } else {
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[wave][db][lane] = c.o[db];
    if (lane < 16) {
      ml[wave][0][lane] = c.m;
      ml[wave][1][lane] = c.l;
    }
    __syncthreads();
    float w[NW];
    m = NEG_BIG;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) m = fmaxf(m, ml[i][0][lane & 15]);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      w[i] = fast_exp2(ml[i][0][lane & 15] - m);
      l += w[i] * ml[i][1][lane & 15];
    }
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      o[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (wave * MINE + k < DB)
#pragma unroll
        for (int i = 0; i < NW; ++i) o[k] += w[i] * acc[i][wave * MINE + k][lane];
    }
  }
  if (it.state >= 0) {
    // units with the same rows leave what they have, the last of them to arrive joins it, in the order of the pages
    const unsigned n = (unsigned)it.group >> WINDOW_STATE_BITS, state0 = (unsigned)it.group & ((1u << WINDOW_STATE_BITS) - 1);
    const __amdgpu_buffer_rsrc_t rs = join_dev::parts_of(a.parts);
    constexpr unsigned PART = (DB + 1) * 1024;  // bytes
    const unsigned mine = ((unsigned)it.state * hkv + kvh) * PART + lane * 16, first = (state0 * hkv + kvh) * PART + lane * 16, step = hkv * PART;
    if (ok)
#pragma unroll
      for (int k = 0; k < MINE; ++k)
        if (wave * MINE + k < DB) join_dev::put_part(rs, mine + (wave * MINE + k) * 1024, o[k]);
    if (wave == 0 && lane < 16) join_dev::put_part(rs, mine + DB * 1024, f32x4_t{m, l, 0.f, 0.f});
    if (!join_dev::last_of(a.counters + (size_t)state0 * hkv + kvh, n, flag)) return;
#pragma unroll
    for (int k = 0; k < MINE; ++k) o[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m = NEG_BIG;
    l = 0.f;
    if (ok) {
      constexpr int B = Pages::joined(MINE);  // states on the way
      for (unsigned p = 0; p < n; p += B) {
        f32x4_t s[B], v[B][MINE];
#pragma unroll
        for (int u = 0; u < B; ++u) {
          const unsigned at = first + min(p + u, n - 1) * step;
          s[u] = join_dev::get_part(rs, at - (lane & 48) * 16 + DB * 1024);
#pragma unroll
          for (int k = 0; k < MINE; ++k) v[u][k] = join_dev::get_part(rs, at + min(wave * MINE + k, DB - 1) * 1024);
        }
        float m_new = m;
#pragma unroll
        for (int u = 0; u < B; ++u) m_new = fmaxf(m_new, s[u][0]);
        const float alpha = fast_exp2(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int k = 0; k < MINE; ++k) o[k] *= alpha;
#pragma unroll
        for (int u = 0; u < B; ++u) {
          const float w = p + u < n ? fast_exp2(s[u][0] - m) : 0.f;
          l += w * s[u][1];
#pragma unroll
          for (int k = 0; k < MINE; ++k) o[k] += w * v[u][k];
        }
      }
    }
  }
  if (ok)
#pragma unroll
    for (int k = 0; k < MINE; ++k)
      if (wave * MINE + k < DB) store_quad(a, it, col_head, col, DH, lane, wave * MINE + k, o[k], l);
}

}  // namespace window_dev
}  // namespace bs
