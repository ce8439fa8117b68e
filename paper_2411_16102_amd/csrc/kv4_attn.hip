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

// calls f with 0, 1 .. N - 1 as constants
template <class F, int... I>
__device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F &&f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

// lane N of each sixteen, in all of them
template <int N>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x150 + N, 0xF, 0xF, true);
}
template <int N>
__device__ __forceinline__ float from_lane(float v) {
  return __uint_as_float(from_lane<N>(__float_as_uint(v)));
}

// c + (lane N of each sixteen's v) x in one instruction, which the compiler does not make of the two.  It does not see either that a lane's register
// must have been written two wait states before another lane reads it: v passes through settled() when it has been written.
template <int N>
__device__ __forceinline__ float add_from_lane(float c, float v, float x) {
  asm("v_fmac_f32_dpp %0, %1, %2 row_newbcast:%3 row_mask:0xf bank_mask:0xf" : "+v"(c) : "v"(v), "v"(x), "n"(N));
  return c;
}
__device__ __forceinline__ void settled(float (&v)[8]) {
  asm volatile("s_nop 1" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
}

// The columns of a unit as in window_device.hpp, on codes.  A value is mid + scale (code - 8), with numbers for each token and group g of channels, so
//   score_t  = sum over g of scale_tg (q_g . (code_tg - 8)) + mid_tg sum(q_g)
//   output_c = sum over t of (p_t scale_tg) (code_tc - 8) + p_t mid_tg
// and no code is ever multiplied by its scale: products take bf16 numbers 16 + code, three operations for two of them, and the rest is done to
// scores and probabilities.  24 sum(q_g) less is where the accumulators of scores begin; 24 sum of p scale is taken off, and p mid
// added, by two products a group whose other operand is the same for all channels.  Rounded are the probabilities, with and without
// scale, to bf16 (at most 2^-9 of the sum of p (8 scale + |mid|)).
template <int DH, int GROUP>
struct FourBitPages {
  static constexpr int KC = DH / 32, DB = DH / 16, NG = DH / GROUP, STEPS = GROUP / 32, BLOCKS = GROUP / 16;
  f32x4_t common[NG];  // of all channels of a group
  float q_sum[NG];
  Unpack unpack;

  __device__ __forceinline__ explicit FourBitPages(const bf16x8_t (&qf)[KC]) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      common[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
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

  // pages [pg0, pg1) of the unit, at most 64
  __device__ __forceinline__ void walk(const WindowArgs &a, const WindowItem &it, int kvh, int lane, int pg0, int pg1, const bf16x8_t (&qf)[KC], Columns<DH> &c) {
    constexpr int KW = DH / 64, VW = DH / 64;  // 16-byte loads of keys and of values
    const int hkv = a.s.n_kv_heads, grp = a.s.n_q_heads / hkv;
    const int jq = lane & 15, g4 = lane >> 4;
    constexpr size_t HEAD = kv4_head_bytes(DH, GROUP);
    const float sc = a.s.scale_log2e;
    const bool ok = jq < it.n_rows * grp;
    const int j = ok ? jq / grp : 0;
    // places are counted from this wavefront's first page
    const int n_pg = pg1 - pg0, first = it.at - 16 * pg0, last = first + it.n_rows - 1, at = first + j, sinks = it.sinks - 16 * pg0;
    const int my_page = a.item_pages[it.page_off + pg0 + min(lane, n_pg - 1)];  // lane i holds page i
    struct Frags {
      u32x4_t k[KW], v[VW], numbers;
    };
    const unsigned char *pool = reinterpret_cast<const unsigned char *>(a.kv_pool) + (size_t)kvh * HEAD;
    const unsigned char *k_base = pool + 4 * kv4_keys_at(g4, jq & 7, 0, 0, DH), *v_base = pool + 4 * kv4_values_at(g4 & 1, jq, DH);
    const unsigned char *n_base = pool + 16 * DH + (g4 & 1) * 64 * NG + jq % (4 * NG) * 16;  // (kind, group) jq of this lane's eight tokens
    const uint32_t page_bytes = (uint32_t)hkv * (uint32_t)HEAD;
    auto load = [&](int pr, Frags &f) __attribute__((always_inline)) {  // (past the end: the last page again, not used)
      const uint32_t p0 = __builtin_amdgcn_readlane(my_page, min(2 * pr, n_pg - 1)), p1 = __builtin_amdgcn_readlane(my_page, min(2 * pr + 1, n_pg - 1));
      const uint64_t k_at = (uint64_t)(jq < 8 ? p0 : p1) * page_bytes, v_at = (uint64_t)(g4 < 2 ? p0 : p1) * page_bytes;
      f.numbers = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(n_base + v_at));
#pragma unroll
      for (int i = 0; i < KW; ++i) f.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(k_base + k_at) + i);
#pragma unroll
      for (int i = 0; i < VW; ++i) f.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(v_base + v_at) + i);
    };
    auto compute = [&](int pr, Frags &f) __attribute__((always_inline)) {
      const int tb = 32 * pr;  // (a pair past the end is masked whole: an early way out would cost copies of all accumulators)
      const int u0 = tb + 8 * g4;  // this lane's eight tokens
      // (Masks are for few pairs.  What passes through an empty asm stays in its branch: left alone, the compiler computes all of them for every pair.)
      const bool whole = tb + 32 <= 16 * n_pg && tb + 31 <= first && (tb > last - a.window || tb + 32 <= sinks);
      if (!whole) {  // wave-uniform: the numbers of tokens that no row sees (the codes of such tokens are numbers whatever their bits)
        int u = u0;
        asm volatile("" : "+v"(f.numbers), "+v"(u));
        const int end = min(16 * n_pg, last + 1), unseen = first - a.window + 1;
        f.numbers = mask_between8(mask_tokens8(f.numbers, u, end), u, sinks, unseen);
      }
      float num[8];  // a kind and group of this lane's tokens
#pragma unroll
      for (int r = 0; r < 8; ++r) num[r] = __uint_as_float(r & 1 ? f.numbers[r >> 1] & 0xFFFF0000u : f.numbers[r >> 1] << 16);
      settled(num);
      float sv[8];
      f32x4_t s[NG][2];
#pragma unroll
      for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int w = i * KC + g * STEPS + k;
            const float from = -CENTRE * q_sum[g];
            s[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(unpack(f.k[w >> 2][w & 3])), qf[g * STEPS + k],
                                                              k == 0 ? f32x4_t{from, from, from, from} : s[g][i], 0, 0, 0);
          }
      each<NG>([&](auto g_) __attribute__((always_inline)) {
        constexpr int g = decltype(g_)::value;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float x = from_lane<g>(num[r]) * s[g][r >> 2][r & 3];
          sv[r] = add_from_lane<NG + g>(g == 0 ? x : sv[r] + x, num[r], q_sum[g]);
        }
      });
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
        for (int g = 0; g < NG; ++g) common[g] *= alpha;
      }
      float ps = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        sv[r] = fast_exp2(__builtin_fmaf(sv[r], sc, -c.m));
        ps += sv[r];
      }
      c.l += ps;
      const bf16x8_t p = as_bf16x8(u32x4_t{pack_bf16x2(sv[0], sv[1]), pack_bf16x2(sv[2], sv[3]), pack_bf16x2(sv[4], sv[5]), pack_bf16x2(sv[6], sv[7])});
      const uint32_t less = 0xC1C0C1C0u;  // -24 twice
      each<NG>([&](auto g_) __attribute__((always_inline)) {
        constexpr int g = decltype(g_)::value;
        float x[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) x[r] = from_lane<2 * NG + g>(num[r]) * sv[r];
        const bf16x8_t px = as_bf16x8(u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])});
        const u32x4_t mid = {from_lane<3 * NG + g>(f.numbers.x), from_lane<3 * NG + g>(f.numbers.y), from_lane<3 * NG + g>(f.numbers.z), from_lane<3 * NG + g>(f.numbers.w)};
        common[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(mid), p, common[g], 0, 0, 0);
        common[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u32x4_t{less, less, less, less}), px, common[g], 0, 0, 0);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          const int db = g * BLOCKS + b;
          c.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(unpack(f.v[db >> 2][db & 3])), px, c.o[db], 0, 0, 0);
        }
      });
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

  __device__ __forceinline__ void finish(Columns<DH> &c) {
#pragma unroll
    for (int db = 0; db < DB; ++db) c.o[db] += common[db / BLOCKS];
  }
};

template <int DH, int GROUP, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void window_unit4_kernel(const WindowArgs a) {
  __shared__ __align__(16) unsigned char lds[WINDOW_UNIT_LDS(DH, NW)];
  window_unit<DH, NW, FourBitPages<DH, GROUP>>(a, blockIdx.x, lds);
}

template <int DH, int GROUP>
hipError_t launch_units4(const WindowArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)a.n_items * (unsigned)a.s.n_kv_heads), block(64 * a.waves);
  if (a.waves == 1) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, 1>), grid, block, 0, stream, a);
  else if (a.waves == 2) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, 2>), grid, block, 0, stream, a);
  else if (a.waves == 4) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, 4>), grid, block, 0, stream, a);
  else if (a.waves == 8) hipLaunchKernelGGL((window_unit4_kernel<DH, GROUP, 8>), grid, block, 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
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
