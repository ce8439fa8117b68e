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
template <int DH, int GROUP, int HEADS_>
struct FourBitPages {
  static constexpr int HEADS = HEADS_, CPH = 16 / HEADS;
  static constexpr int KC = DH / 32, DB = DH / 16, NG = DH / GROUP, STEPS = GROUP / 32, BLOCKS = GROUP / 16;
  static constexpr int joined(int blocks) { return blocks <= 1 ? 8 : blocks <= 4 ? 4 : 2; }
  bf16x8_t q[HEADS][KC];
  f32x4_t common[NG];  // of all channels of a group
  float q_sum[NG], mids[NG];
  Unpack unpack;

  __device__ __forceinline__ explicit FourBitPages(const bf16x8_t (&qf)[KC]) {
    const int mine = (threadIdx.x & 15) / CPH;
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        u32x4_t v = __builtin_bit_cast(u32x4_t, qf[i]);
        if (HEADS > 1 && mine != h) v = u32x4_t{0u, 0u, 0u, 0u};
        q[h][i] = as_bf16x8(v);
      }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      common[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      mids[g] = 0.f;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += (float)qf[g * STEPS + i][k];
      s += __shfl_xor(s, 16, 64);
      s += __shfl_xor(s, 32, 64);
      q_sum[g] = s;
    }
  }

  // pages [pg0, pg1) of the unit, at most 64, of KV heads kvh ..
  __device__ __forceinline__ void walk(const WindowArgs &a, const WindowItem &it, int kvh, int lane, int pg0, int pg1, const bf16x8_t (&)[KC], Columns<DH> &c) {
    constexpr int KW = DH / 64, VW = DH / 64;  // 16-byte loads of a head's keys and of its values
    constexpr int HEAD = kv4_head_bytes(DH, GROUP);
    const int hkv = a.s.n_kv_heads, grp = a.s.n_q_heads / hkv;
    const int jq = lane & 15, g4 = lane >> 4, col = jq % CPH, mine = jq / CPH;
    const float sc = a.s.scale_log2e;
    const int j = col < it.n_rows * grp ? col / grp : 0;
    // places are counted from this wavefront's first page
    const int n_pg = pg1 - pg0, first = it.at - 16 * pg0, last = first + it.n_rows - 1, at = first + j, sinks = it.sinks - 16 * pg0;
    const int my_page = a.item_pages[it.page_off + pg0 + min(lane, n_pg - 1)];  // lane i holds page i
    const unsigned char *pool = reinterpret_cast<const unsigned char *>(a.kv_pool) + (size_t)kvh * HEAD;
    const unsigned char *k_base = pool + 4 * kv4_keys_at(g4, jq & 7, 0, 0, DH), *v_base = pool + 4 * kv4_values_at(g4 & 1, jq, DH);
    const unsigned char *n_base = pool + (size_t)mine * HEAD + kv4_number_at(8 * (g4 & 1), jq & 3, 0, DH, GROUP);  // kind jq % 4 of this lane's eight tokens
    const uint32_t page_bytes = (uint32_t)hkv * (uint32_t)HEAD;
    u32x4_t k[HEADS][KW], v[HEADS][VW], numbers[NG];
    // (past the end: the last page again, not used)
    auto page = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane(my_page, min(i, n_pg - 1)); };
    auto load_keys = [&](int pr) __attribute__((always_inline)) {
      const uint32_t p0 = page(2 * pr), p1 = page(2 * pr + 1);
      const unsigned char *n_at = n_base + (uint64_t)(g4 < 2 ? p0 : p1) * page_bytes, *k_at = k_base + (uint64_t)(jq < 8 ? p0 : p1) * page_bytes;
#pragma unroll
      for (int g = 0; g < NG; ++g) numbers[g] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(n_at) + 4 * g);
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int i = 0; i < KW; ++i) k[h][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(k_at + h * HEAD) + 32 * i);
    };
    auto load_values = [&](int pr) __attribute__((always_inline)) {
      const uint32_t p0 = page(2 * pr), p1 = page(2 * pr + 1);
      const unsigned char *v_at = v_base + (uint64_t)(g4 < 2 ? p0 : p1) * page_bytes;
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int i = 0; i < VW; ++i) v[h][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(v_at + h * HEAD) + 32 * i);
    };
    load_keys(0);
    load_values(0);
    for (int pr = 0; 2 * pr < n_pg; ++pr) {
      const int tb = 32 * pr, u0 = tb + 8 * g4;  // this lane's eight tokens
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
      // (four accumulators in turn at least: a product that goes on from the last one's result waits for it)
      constexpr int TURNS = NG == 1 ? 2 : 1;
      f32x4_t s[NG][TURNS][2];
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float from = -CENTRE * q_sum[g];
          s[g][0][i] = f32x4_t{from, from, from, from};
          if constexpr (TURNS == 2) s[g][1][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int n = 0; n < STEPS; ++n)
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int w = i * KC + g * STEPS + n;
              f32x4_t &to = s[g][(h * STEPS + n) % TURNS][i];
              to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(unpack(k[h][w >> 2][w & 3])), q[h][g * STEPS + n], to, 0, 0, 0);
              __builtin_amdgcn_sched_barrier(0x7F6);  // (in this order; all but matrix instructions may move)
            }
      float sv[8];
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          float d = s[g][0][r >> 2][r & 3];
          if constexpr (TURNS == 2) d += s[g][1][r >> 2][r & 3];
          const float x = of_quad<0>(num[g][r]) * d;
          sv[r] = add_of_quad<1>(g == 0 ? x : sv[r] + x, num[g][r], q_sum[g]);
        }
      load_keys(pr + 1);
      if (!whole) {
        int from = u0;
        asm volatile("" : "+v"(sv[0]), "+v"(sv[1]), "+v"(sv[2]), "+v"(sv[3]), "+v"(sv[4]), "+v"(sv[5]), "+v"(sv[6]), "+v"(sv[7]), "+v"(from));
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const int u = from + r;  // (one condition, selected by: see window_device.hpp)
          const bool hidden = (u > at) | ((u <= at - a.window) & (u >= sinks)) | (u >= 16 * n_pg);
          sv[r] = hidden ? -INFINITY : sv[r];
        }
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
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          common[g] *= alpha;
          mids[g] *= alpha;
        }
      }
      float ps = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        sv[r] = fast_exp2(__builtin_fmaf(sv[r], sc, -c.m));
        ps += sv[r];
      }
      c.l += ps;
      const uint32_t less = 0xC1C0C1C0u;  // -24 twice
      u32x4_t px[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float x[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          x[r] = of_quad<2>(num[g][r]) * sv[r];
          mids[g] = add_of_quad<3>(mids[g], num[g][r], sv[r]);
        }
        px[g] = u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        common[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u32x4_t{less, less, less, less}), as_bf16x8(px[g]), common[g], 0, 0, 0);
      }
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          u32x4_t own = px[g];
          if constexpr (HEADS > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) own[i] = mine == h ? px[g][i] : 0u;
          }
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            const int db = g * BLOCKS + b;
            c.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(unpack(v[h][db >> 2][db & 3])), as_bf16x8(own), c.o[db], 0, 0, 0);
          }
        }
      load_values(pr + 1);
    }
  }

  __device__ __forceinline__ void finish(Columns<DH> &c) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      mids[g] += __shfl_xor(mids[g], 16, 64);
      mids[g] += __shfl_xor(mids[g], 32, 64);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) c.o[db] += common[db / BLOCKS] + mids[db / BLOCKS];
  }
};

// wavefronts that the registers of a SIMD hold
constexpr int resident(int dh, int group, int heads) { return dh == 128 ? (heads == 2 || group == 32 ? 2 : 3) : heads == 2 ? 3 : 4; }
template <int DH, int GROUP, int HEADS, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(resident(DH, GROUP, HEADS), resident(DH, GROUP, HEADS)))) void window_unit4_kernel(const WindowArgs a) {
  __shared__ __align__(16) unsigned char lds[WINDOW_UNIT_LDS(DH, NW)];
  window_unit<DH, NW, FourBitPages<DH, GROUP, HEADS>>(a, blockIdx.x, lds);
}

template <int DH, int GROUP, int HEADS>
hipError_t launch_heads4(const WindowArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)a.n_items * (unsigned)(a.s.n_kv_heads / HEADS)), block(64 * a.waves);
  if (a.waves == 1) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 1>), grid, block, 0, stream, a);
  else if (a.waves == 2) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 2>), grid, block, 0, stream, a);
  else if (a.waves == 4) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 4>), grid, block, 0, stream, a);
  else if (a.waves == 8) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, HEADS, 8>), grid, block, 0, stream, a);
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
