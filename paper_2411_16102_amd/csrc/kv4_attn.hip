// Window attention's narrow work over a cache in four bits.
#include <type_traits>
#include <utility>

#include "kv4.hpp"
#include "kv4_device.hpp"
#include "window_device.hpp"

namespace bs {
namespace {
using namespace kv4_dev;
using namespace window_dev;

// lane N of each four lanes, in all of them
template <int N>
__device__ __forceinline__ float of_quad(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x55 * N, 0xF, 0xF, true));
}
// c + (lane N of each four's v) x in one instruction, which the compiler does not make of the two.  It does not see either that a lane's register
// must have been written two wait states before another lane reads it: v passes through settled() when it has been written.
template <int N>
__device__ __forceinline__ float add_of_quad(float c, float v, float x) {
  asm("v_fmac_f32_dpp %0, %1, %2 quad_perm:[%3,%3,%3,%3] row_mask:0xf bank_mask:0xf" : "+v"(c) : "v"(v), "v"(x), "n"(N));
  return c;
}
__device__ __forceinline__ void settled(float (&v)[8]) {
  asm volatile("s_nop 1" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
}

// The columns of a unit as in window_device.hpp, on codes.  A value is mid + scale (code - 8), with numbers for each token and group g of channels, so
//   score_t  = sum over g of scale_tg (q_g . (code_tg - 8)) + mid_tg sum(q_g)
//   output_c = sum over t of (p_t scale_tg) (code_tc - 8) + p_t mid_tg
// and no code is ever multiplied by its scale: products take bf16 numbers 16 + code, seven operations for eight of them, and the rest is done to
// scores and probabilities.  24 sum(q_g) less is where the accumulators of scores begin, 24 sum of p scale is taken off by a product a
// group whose other operand is the same for all channels, and sum of p mid is one number a column and group, kept in 32 bits.  Rounded are the
// probabilities times scale, to bf16 (at most 2^-9 of the sum of p 8 scale).
//
// A single token has few columns, its heads of a KV group, and scores and probabilities cost as much for sixteen: so HEADS KV heads share a wavefront, 16 / HEADS
// columns each.  Columns of other heads are zero in a head's queries, so that the products of all heads add up in the same accumulators,
// and in its probabilities.  A lane's numbers are those of its column's head: four lanes have the four kinds (scale and mid of keys, of values) of
// a group in one load, and take them from one another.
//
// The rows of a longer segment share their pages too: BLOCKS blocks of sixteen columns to a wavefront, and four wavefronts for which a code is brought
// to 16 + code once.
template <int DH, int GROUP, int HEADS, int BLOCKS>
struct FourBits {
  static_assert(HEADS == 1 || BLOCKS == 1, "columns of several heads, or several blocks of them");
  static constexpr int CPH = 16 / HEADS, KC = DH / 32, DB = DH / 16, NG = DH / GROUP, STEPS = GROUP / 32, PER = GROUP / 16;
  // What brings a third wavefront of several blocks to a SIMD: queries in LDS, and, beside those of 128 channels, codes once instead of twice.
  static constexpr bool Q_LDS = BLOCKS > 1 && ((DH == 128 && GROUP == 128) || (DH == 64 && GROUP == 32)), TWICE = !Q_LDS || DH == 64;
  static constexpr int WAVES = DH == 128 && GROUP == 64 ? 2 : 3;  // of several blocks, on a SIMD
  typedef __attribute__((address_space(3))) bf16x8_t Lds;
  bf16x8_t q[Q_LDS ? 1 : HEADS * BLOCKS][KC];
  Lds *q_lds;  // this lane's, [block][32 channels], 64 apart
  f32x4_t common[BLOCKS][NG];  // of all channels of a group
  float q_sum[BLOCKS][NG], mids[BLOCKS][NG];
  Unpack unpack;

  __device__ __forceinline__ void begin(int b, const bf16x8_t (&qf)[KC]) {
    const int mine = (threadIdx.x & 15) / CPH;
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        u32x4_t v = __builtin_bit_cast(u32x4_t, qf[i]);
        if (HEADS > 1 && mine != h) v = u32x4_t{0u, 0u, 0u, 0u};
        if constexpr (Q_LDS) q_lds[(b * KC + i) * 64] = as_bf16x8(v);
        else q[h + b][i] = as_bf16x8(v);
      }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      common[b][g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      mids[b][g] = 0.f;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += (float)qf[g * STEPS + i][k];
      s += __shfl_xor(s, 16, 64);
      s += __shfl_xor(s, 32, 64);
      q_sum[b][g] = s;
    }
  }

  // A pair of pages, places tb .. tb + 31 of n_pg pages: scores, probabilities and sums of all columns.  numbers: of this lane's eight tokens;
  // keys(h, w), values(h, db): codes as bf16; then(): once numbers and keys are done with.
  template <class Keys, class Values, class Then>
  __device__ __forceinline__ void pair(const WindowArgs &a, int tb, int n_pg, int first, int last, int sinks, const int (&at)[BLOCKS], u32x4_t (&numbers)[NG],
                                       Columns<DH> (&c)[BLOCKS], Keys &&keys, Values &&values, Then &&then) {
    const float sc = a.s.scale_log2e;
    const int u0 = tb + 8 * ((threadIdx.x & 63) >> 4), mine = (threadIdx.x & 15) / CPH;  // this lane's eight tokens; its column's head
    // (Masks are for few pairs.  What passes through an empty asm stays in its branch: left alone, the compiler computes all of them for every pair.)
    const bool whole = tb + 32 <= 16 * n_pg && tb + 31 <= first && (tb > last - a.window || tb + 32 <= sinks);
    if (!whole) {  // wave-uniform: the numbers of tokens that no row sees (the codes of such tokens are numbers whatever their bits)
      int u = u0;
      asm volatile("" : "+v"(u));
      const int end = min(16 * n_pg, last + 1), unseen = first - a.window + 1;
#pragma unroll
      for (int g = 0; g < NG; ++g) numbers[g] = mask_between8(mask_tokens8(numbers[g], u, end), u, sinks, unseen);
    }
    float num[NG][8];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
#pragma unroll
      for (int r = 0; r < 8; ++r) num[g][r] = __uint_as_float(r & 1 ? numbers[g][r >> 1] & 0xFFFF0000u : numbers[g][r >> 1] << 16);
      settled(num[g]);
    }
    // scores, some groups of channels at a time; four accumulators in turn at least: a product that goes on from the last one's result waits for it
    constexpr int GS = BLOCKS == 1 && NG >= 2 ? NG : 1, TURNS = BLOCKS == 1 && GS == 1 ? 2 : 1;
    const Lds *q_now = q_lds;
    if constexpr (Q_LDS) asm volatile("" : "+v"(q_now));  // (read here every time)
    float sv[BLOCKS][8];
#pragma unroll
    for (int g0 = 0; g0 < NG; g0 += GS) {
      f32x4_t s[GS][TURNS][BLOCKS][2];
#pragma unroll
      for (int g = 0; g < GS; ++g)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float from = -CENTRE * q_sum[b][g0 + g];
            s[g][0][b][i] = f32x4_t{from, from, from, from};
            if constexpr (TURNS == 2) s[g][1][b][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          }
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int n = 0; n < STEPS; ++n)
#pragma unroll
          for (int g = 0; g < GS; ++g) {
            const int step = (g0 + g) * STEPS + n;
            bf16x8_t qs[BLOCKS];
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
              if constexpr (Q_LDS) qs[b] = q_now[(b * KC + step) * 64];
              else qs[b] = q[h + b][step];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const bf16x8_t codes = keys(h, i * KC + step);
#pragma unroll
              for (int b = 0; b < BLOCKS; ++b) {
                f32x4_t &to = s[g][(h * STEPS + n) % TURNS][b][i];
                to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes, qs[b], to, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0x7F6);  // (in this order; all but matrix instructions may move)
              }
            }
          }
#pragma unroll
      for (int g = 0; g < GS; ++g)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            float d = s[g][0][b][r >> 2][r & 3];
            if constexpr (TURNS == 2) d += s[g][1][b][r >> 2][r & 3];
            const float x = of_quad<0>(num[g0 + g][r]) * d;
            sv[b][r] = add_of_quad<1>(g0 + g == 0 ? x : sv[b][r] + x, num[g0 + g][r], q_sum[b][g0 + g]);
          }
    }
    then();
    if (!whole) {
      int from = u0;
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        float(&sb)[8] = sv[b];
        asm volatile("" : "+v"(sb[0]), "+v"(sb[1]), "+v"(sb[2]), "+v"(sb[3]), "+v"(sb[4]), "+v"(sb[5]), "+v"(sb[6]), "+v"(sb[7]), "+v"(from));
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const int u = from + r;  // (one condition, selected by: see window_device.hpp)
          const bool hidden = (u > at[b]) | ((u <= at[b] - a.window) & (u >= sinks)) | (u >= 16 * n_pg);
          sb[r] = hidden ? -INFINITY : sb[r];
        }
      }
    }
    float mx[BLOCKS];
    bool moves = false;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const float(&sb)[8] = sv[b];
      mx[b] = sc * fmaxf(fmaxf(fmaxf(sb[0], sb[1]), fmaxf(sb[2], sb[3])), fmaxf(fmaxf(sb[4], sb[5]), fmaxf(sb[6], sb[7])));
      moves |= mx[b] > c[b].m + TAU;
    }
    if (__builtin_amdgcn_ballot_w64(moves) != 0) {  // (see TAU: the reference moves rarely)
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        mx[b] = fmaxf(mx[b], __shfl_xor(mx[b], 16, 64));
        mx[b] = fmaxf(mx[b], __shfl_xor(mx[b], 32, 64));
        const float m_new = fmaxf(c[b].m, mx[b]), alpha = fast_exp2(c[b].m - m_new);
        c[b].m = m_new;
        c[b].l *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) c[b].o[db] *= alpha;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          common[b][g] *= alpha;
          mids[b][g] *= alpha;
        }
      }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      float(&sb)[8] = sv[b];
      float ps = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        sb[r] = fast_exp2(__builtin_fmaf(sb[r], sc, -c[b].m));
        ps += sb[r];
      }
      c[b].l += ps;
    }
    u32x4_t px[BLOCKS];  // probabilities times scale
    auto scaled = [&](int b, int g) __attribute__((always_inline)) {
      const uint32_t less = 0xC1C0C1C0u;  // -24 twice
      float x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        x[r] = of_quad<2>(num[g][r]) * sv[b][r];
        mids[b][g] = add_of_quad<3>(mids[b][g], num[g][r], sv[b][r]);
      }
      px[b] = u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
      common[b][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u32x4_t{less, less, less, less}), as_bf16x8(px[b]), common[b][g], 0, 0, 0);
    };
    if constexpr (HEADS == 1) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) scaled(b, g);
#pragma unroll
        for (int n = 0; n < PER; ++n) {
          const int db = g * PER + n;
          const bf16x8_t codes = values(0, db);
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) c[b].o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes, as_bf16x8(px[b]), c[b].o[db], 0, 0, 0);
        }
      }
    } else {
      u32x4_t all[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        scaled(0, g);
        all[g] = px[0];
      }
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          u32x4_t own;
#pragma unroll
          for (int i = 0; i < 4; ++i) own[i] = mine == h ? all[db / PER][i] : 0u;
          c[0].o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values(h, db), as_bf16x8(own), c[0].o[db], 0, 0, 0);
        }
    }
  }

  // one block of columns, pages [pg0, pg1) of the unit, at most 64, of KV heads kvh ..
  __device__ __forceinline__ void walk(const WindowArgs &a, const WindowItem &it, int kvh, int lane, int pg0, int pg1, Columns<DH> (&c)[1]) {
    constexpr int KW = DH / 64, VW = DH / 64;  // 16-byte loads of a head's keys and of its values
    constexpr int HEAD = kv4_head_bytes(DH, GROUP);
    const int hkv = a.s.n_kv_heads, grp = a.s.n_q_heads / hkv;
    const int jq = lane & 15, g4 = lane >> 4, col = jq % CPH, mine = jq / CPH;
    // places are counted from this wavefront's first page
    const int n_pg = pg1 - pg0, first = it.at - 16 * pg0, last = first + it.n_rows - 1, sinks = it.sinks - 16 * pg0;
    const int at[1] = {first + (col < it.n_rows * grp ? col / grp : 0)};
    const int my_page = a.item_pages[it.page_off + pg0 + min(lane, n_pg - 1)];  // lane i holds page i
    const unsigned char *pool = reinterpret_cast<const unsigned char *>(a.kv_pool) + (size_t)kvh * HEAD;
    const unsigned char *k_base = pool + 4 * kv4_keys_at(g4, jq & 7, 0, 0, DH), *v_base = pool + 4 * kv4_values_at(g4 & 1, jq, DH);
    const unsigned char *n_base = pool + (size_t)mine * HEAD + kv4_number_at(8 * (g4 & 1), jq & 3, 0, DH, GROUP);  // kind jq % 4 of this lane's eight tokens
    const uint32_t page_bytes = (uint32_t)hkv * (uint32_t)HEAD;
    u32x4_t k[HEADS][KW], v[HEADS][VW], numbers[NG];
    auto ask = [](const unsigned char *p) __attribute__((always_inline)) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p)); };
    // (past the end: the last page again, not used)
    auto page = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane(my_page, min(i, n_pg - 1)); };
    auto load_keys = [&](int pr) __attribute__((always_inline)) {
      const uint32_t p0 = page(2 * pr), p1 = page(2 * pr + 1);
      const unsigned char *n_at = n_base + (uint64_t)(g4 < 2 ? p0 : p1) * page_bytes, *k_at = k_base + (uint64_t)(jq < 8 ? p0 : p1) * page_bytes;
#pragma unroll
      for (int g = 0; g < NG; ++g) numbers[g] = ask(n_at + 64 * g);
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int i = 0; i < KW; ++i) k[h][i] = ask(k_at + h * HEAD + 512 * i);
    };
    auto load_values = [&](int pr) __attribute__((always_inline)) {
      const uint32_t p0 = page(2 * pr), p1 = page(2 * pr + 1);
      const unsigned char *v_at = v_base + (uint64_t)(g4 < 2 ? p0 : p1) * page_bytes;
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int i = 0; i < VW; ++i) v[h][i] = ask(v_at + h * HEAD + 512 * i);
    };
    load_keys(0);
    load_values(0);
    for (int pr = 0; 2 * pr < n_pg; ++pr) {
      pair(
          a, 32 * pr, n_pg, first, last, sinks, at, numbers, c, [&](int h, int w) __attribute__((always_inline)) { return as_bf16x8(unpack(k[h][w >> 2][w & 3])); },
          [&](int h, int db) __attribute__((always_inline)) { return as_bf16x8(unpack(v[h][db >> 2][db & 3])); }, [&]() __attribute__((always_inline)) { load_keys(pr + 1); });
      load_values(pr + 1);
    }
  }

  // Pages [pg0, pg1) of an item, at most 64, of KV head kvh, for the four wavefronts of a workgroup, whose rows are it's from row `from` on, n_rows of them.  Each brings a
  // quarter of the codes of the next pair to LDS as bf16, in the order in which products take them: [keys, values][operand][lane], twice; or once,
  // keys when all have read the last pair's and values when they have read those.
  __device__ __forceinline__ void walk_shared(const WindowArgs &a, const WindowItem &it, int from, int n_rows, int kvh, int lane, int wave, int pg0, int pg1, u32x4_t *lds,
                                              Columns<DH> (&c)[BLOCKS]) {
    constexpr int HEAD = kv4_head_bytes(DH, GROUP), W = DH / 32, OPERANDS = DH / 16;  // W: words of a thread; operands of keys, of values
    const int hkv = a.s.n_kv_heads, grp = a.s.n_q_heads / hkv;
    const int jq = lane & 15, g4 = lane >> 4;
    const int n_pg = pg1 - pg0, first = it.at + from - 16 * pg0, last = first + n_rows - 1, sinks = it.sinks - 16 * pg0;
    int at[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) at[b] = first + (16 * b + jq < n_rows * grp ? (16 * b + jq) / grp : 0);
    const int my_page = a.item_pages[it.page_off + pg0 + min(lane, n_pg - 1)];  // lane i holds page i
    const unsigned char *pool = reinterpret_cast<const unsigned char *>(a.kv_pool) + (size_t)kvh * HEAD;
    // wavefronts 0 and 1 take keys, 2 and 3 values: of the sixteen bytes of a lane's first load all, or all of its second; or a half each
    const bool values = wave >= 2;
    const int part = wave & 1, word0 = part * W;
    const unsigned char *c_base = pool + 4 * (values ? kv4_values_at(g4 & 1, jq, DH) : kv4_keys_at(g4, jq & 7, 0, 0, DH)) + (DH == 128 ? 512 * part : 8 * part);
    const unsigned char *n_base = pool + kv4_number_at(8 * (g4 & 1), jq & 3, 0, DH, GROUP);
    const bool second = values ? g4 >= 2 : jq >= 8;  // of this lane's codes: of the pair's second page
    const uint32_t page_bytes = (uint32_t)hkv * (uint32_t)HEAD;
    uint32_t codes[W];
    u32x4_t numbers[NG];
    // (past the end: the last page again, not used)
    auto page = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane(my_page, min(i, n_pg - 1)); };
    auto load_codes = [&](int pr) __attribute__((always_inline)) {
      const uint32_t p0 = page(2 * pr), p1 = page(2 * pr + 1);
      const unsigned char *p = c_base + (uint64_t)(second ? p1 : p0) * page_bytes;
      if constexpr (W == 4) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t *>(p);
#pragma unroll
        for (int i = 0; i < W; ++i) codes[i] = x[i];
      } else {
        const u32x2_t x = *reinterpret_cast<const u32x2_t *>(p);
#pragma unroll
        for (int i = 0; i < W; ++i) codes[i] = x[i];
      }
    };
    auto load_numbers = [&](int pr) __attribute__((always_inline)) {
      const unsigned char *p = n_base + (uint64_t)(g4 < 2 ? page(2 * pr) : page(2 * pr + 1)) * page_bytes;
#pragma unroll
      for (int g = 0; g < NG; ++g) numbers[g] = *reinterpret_cast<const u32x4_t *>(p + 64 * g);
    };
    auto put = [&](int pr) __attribute__((always_inline)) {
      u32x4_t *to = lds + ((TWICE ? pr & 1 : 0) * 2 + values) * OPERANDS * 64 + word0 * 64 + lane;
#pragma unroll
      for (int i = 0; i < W; ++i) to[i * 64] = unpack(codes[i]);
    };
    auto meet = []() __attribute__((always_inline)) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0xC07F);  // (LDS alone; where loads are waited for is said at window_rows4_kernel)
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    load_codes(0);
    load_numbers(0);
    put(0);
    load_codes(1);
    meet();
    for (int pr = 0; 2 * pr < n_pg; ++pr) {
      if constexpr (TWICE) {
        put(pr + 1);
        load_codes(pr + 2);
      }
      auto keys_read = [&]() __attribute__((always_inline)) {
        load_numbers(pr + 1);
        if constexpr (!TWICE) {
          meet();  // (and this pair's values are there)
          if (!values) {
            put(pr + 1);
            load_codes(pr + 2);
          }
        }
      };
      const int tb = 32 * pr;
      const bool seen = n_rows > 0 && tb <= last && (tb + 31 > first - a.window || tb < sinks);  // wave-uniform
      if (seen) {
        const u32x4_t *own = lds + (TWICE ? pr & 1 : 0) * 2 * OPERANDS * 64 + lane;
        pair(
            a, tb, n_pg, first, last, sinks, at, numbers, c, [&](int, int w) __attribute__((always_inline)) { return as_bf16x8(own[w * 64]); },
            [&](int, int db) __attribute__((always_inline)) { return as_bf16x8(own[(OPERANDS + db) * 64]); }, keys_read);
      } else {
        keys_read();
      }
      meet();  // what was read may be overwritten, what was written is there
      if (!TWICE && values) {
        put(pr + 1);
        load_codes(pr + 2);
      }
    }
  }

  __device__ __forceinline__ void finish(int b, Columns<DH> &c) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      mids[b][g] += __shfl_xor(mids[b][g], 16, 64);
      mids[b][g] += __shfl_xor(mids[b][g], 32, 64);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) c.o[db] += common[b][db / PER] + mids[b][db / PER];
  }
};

// As window_unit walks them: one block of columns.
template <int DH, int GROUP, int HEADS_>
struct FourBitPages : FourBits<DH, GROUP, HEADS_, 1> {
  static constexpr int HEADS = HEADS_;
  static constexpr int joined(int blocks) { return blocks <= 1 ? 8 : blocks <= 4 ? 4 : 2; }
  __device__ __forceinline__ explicit FourBitPages(const bf16x8_t (&qf)[DH / 32]) { this->begin(0, qf); }
  __device__ __forceinline__ void walk(const WindowArgs &a, const WindowItem &it, int kvh, int lane, int pg0, int pg1, const bf16x8_t (&)[DH / 32], Columns<DH> &c) {
    Columns<DH> one[1] = {c};
    FourBits<DH, GROUP, HEADS_, 1>::walk(a, it, kvh, lane, pg0, pg1, one);
    c = one[0];
  }
  __device__ __forceinline__ void finish(Columns<DH> &c) { FourBits<DH, GROUP, HEADS_, 1>::finish(0, c); }
};

// Rows of longer segments: a workgroup per (item, KV head), two blocks of columns to a wavefront, all of the pages that the item's rows see.  Codes are
// brought to bf16 once for the four, which takes 28 vector operations a pair of pages of each instead of 112; 16 reads of LDS give them back.  Bound by
// what a SIMD issues, 230 vector operations and 34 matrix instructions a pair and wavefront (128 channels in one group; of the cycles of CUs at work vector operations take 64 %, matrix
// instructions 29 %), by the last round (below: 1088 workgroups on 768 places), and by loads: once in every pair the compiler waits for all of a wavefront's loads, the codes that it has just
// asked for among them, because pairs that are seen and pairs that are not load their numbers in branches of their own; other wavefronts of the SIMD have to cover that round trip.
// 64-wide heads in two groups keep one register in scratch, around the loop.  Six segments of about 700 rows behind 1500 tokens, 8 KV heads with four
// queries each: 201 us, as narrow work 230.  Slower: two wavefronts on a SIMD (211; of 64-wide heads 185 instead of 159, in two groups 221 instead of 196), every
// wavefront its own codes (224; with three or four blocks and one wavefront a SIMD 319 and 384), one block of columns and four wavefronts (224).  Pages brought to fp16 and bf16 once for the
// kernel of longer segments of a cache in bf16 took 199 us there, but with all batches of its kind 1.4 to 1.8 times the time even of the first of these, and a second copy of the pages.
template <int DH, int GROUP>
using RowBits = FourBits<DH, GROUP, 1, KV4_ROW_BLOCKS>;
template <int DH, int GROUP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RowBits<DH, GROUP>::WAVES, RowBits<DH, GROUP>::WAVES))) void window_rows4_kernel(const WindowArgs a) {
  typedef RowBits<DH, GROUP> Bits;
  constexpr int QUERIES = Bits::Q_LDS ? KV4_ROW_BLOCKS * (DH / 32) * 64 : 1;  // of a wavefront
  const int hkv = a.s.n_kv_heads, grp = a.s.n_q_heads / hkv, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  __shared__ u32x4_t lds[(Bits::TWICE ? 2 : 1) * 2 * (DH / 16) * 64];
  __shared__ bf16x8_t queries[4 * QUERIES];
  const int kvh = blockIdx.x % hkv, rows = max(1, 16 * KV4_ROW_BLOCKS / grp), from = wave * rows;
  const WindowItem it = a.items[blockIdx.x / hkv];
  const int n_rows = max(0, min(rows, it.n_rows - from));
  Bits bits;
  bits.q_lds = (typename Bits::Lds *)(queries + (Bits::Q_LDS ? wave * QUERIES + lane : 0));
  Columns<DH> c[KV4_ROW_BLOCKS];
#pragma unroll
  for (int b = 0; b < KV4_ROW_BLOCKS; ++b) {
    const int col = 16 * b + (lane & 15);
    const bool ok = col < n_rows * grp;
    bf16x8_t qf[DH / 32];
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) {
      u32x4_t v = {0u, 0u, 0u, 0u};
      if (ok) v = ld16(a.q + (it.row0 + from + col / grp) * a.q_stride + (kvh * grp + col % grp) * DH + 32 * i + 8 * (lane >> 4));
      qf[i] = as_bf16x8(v);
    }
    bits.begin(b, qf);
#pragma unroll
    for (int db = 0; db < DH / 16; ++db) c[b].o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    c[b].m = NEG_BIG;
    c[b].l = 0.f;
  }
  for (int pg = 0; pg < it.n_pages; pg += 64) bits.walk_shared(a, it, from, n_rows, kvh, lane, wave, pg, min(pg + 64, it.n_pages), lds, c);
#pragma unroll
  for (int b = 0; b < KV4_ROW_BLOCKS; ++b) {
    bits.finish(b, c[b]);
    float l = c[b].l;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const int col = 16 * b + (lane & 15);
    if (col < n_rows * grp)
#pragma unroll
      for (int db = 0; db < DH / 16; ++db) store_quad(a, it, kvh, from * grp + col, DH, lane, db, c[b].o[db], l);
  }
}

template <int DH, int GROUP, int HEADS, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(kv4_resident(DH, GROUP, HEADS), kv4_resident(DH, GROUP, HEADS)))) void window_unit4_kernel(const WindowArgs a) {
  __shared__ __align__(16) unsigned char lds[WINDOW_UNIT_LDS(DH, NW)];
  window_unit<DH, NW, FourBitPages<DH, GROUP, HEADS>>(a, blockIdx.x, lds);
}

template <int DH, int GROUP, int HEADS>
hipError_t launch_heads4(const WindowArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)a.n_items * (unsigned)(a.s.n_kv_heads / HEADS)), block(64 * a.waves);
  if (a.waves == 1) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 1>), grid, block, 0, stream, a);
  else if (a.waves == 2) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 2>), grid, block, 0, stream, a);
  else if (a.waves == 4) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 4>), grid, block, 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}
template <int DH, int GROUP>
hipError_t launch_units4(const WindowArgs &a, hipStream_t stream) {
  if (a.heads < 1 || a.s.n_kv_heads % a.heads) return hipErrorInvalidValue;
  if (a.heads == 2) return launch_heads4<DH, GROUP, 2>(a, stream);
  return a.heads == 1 ? launch_heads4<DH, GROUP, 1>(a, stream) : hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_window_rows4(const WindowArgs &a, int group, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)a.n_items * (unsigned)a.s.n_kv_heads), block(256);
  if (a.s.head_dim == 128 && group == 128) hipLaunchKernelGGL((window_rows4_kernel<128, 128>), grid, block, 0, stream, a);
  else if (a.s.head_dim == 128 && group == 64) hipLaunchKernelGGL((window_rows4_kernel<128, 64>), grid, block, 0, stream, a);
  else if (a.s.head_dim == 64 && group == 64) hipLaunchKernelGGL((window_rows4_kernel<64, 64>), grid, block, 0, stream, a);
  else if (a.s.head_dim == 64 && group == 32) hipLaunchKernelGGL((window_rows4_kernel<64, 32>), grid, block, 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_window_units4(const WindowArgs &a, int group, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  if (a.s.head_dim == 128 && group == 128) return launch_units4<128, 128>(a, stream);
  if (a.s.head_dim == 128 && group == 64) return launch_units4<128, 64>(a, stream);
  if (a.s.head_dim == 128 && group == 32) return launch_units4<128, 32>(a, stream);
  if (a.s.head_dim == 64 && group == 64) return launch_units4<64, 64>(a, stream);
  if (a.s.head_dim == 64 && group == 32) return launch_units4<64, 32>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace bs
