// Products of few rows with 4-bit weights that have a scale per group of inputs.
//
//   y[m, n] = sum_g scale[n, g] * (sum_{k in g} x[m, k] w[n, k] - zero[n, g] sum_{k in g} x[m, k])
//
// The weights become bf16 matrix operands without arithmetic: 0x4300 | w is the bf16 number 128 + w (its last mantissa
// bit counts 1; integers in the mantissa of a power of two: Kim, Henry, Fahim, Awadalla, "Who Says Elephants Can't Run", 2022), so a
// shift and an and-or make two of them, and
//   sum x w = sum x (128 + w) - 128 sum x,
// which joins the zero point: y += scale * (D - (128 + zero) * X), D the product over the group and X the sum of its x.  All in 32 bits: what that
// leaves in y is 2^-24 of sum |x| (128 + w) |scale| for every step that a term passes through, however small y itself is.  Measured over random x and
// weights the error against 64 bits is that of rounding y, 1.7e-3, as without the offset.
#include <algorithm>

#include "../../include/blendstep_stream.h"
#include "common.hpp"
#include "context.hpp"
#include "join.hpp"
#include "w4.hpp"

using namespace bs;

namespace bs {
namespace {
using namespace join_dev;

// The constants live in registers: as literals they would keep the and and the or apart.
struct Unpack {
  uint32_t mask = 0x000F000Fu, base = 0x43004300u;
  __device__ __forceinline__ Unpack() { asm volatile("" : "+s"(mask), "+v"(base)); }
  __device__ __forceinline__ bf16x8_t operator()(uint32_t w) const {
    const u32x4_t v = {(w & mask) | base, ((w >> 4) & mask) | base, ((w >> 8) & mask) | base, ((w >> 12) & mask) | base};
    return as_bf16x8(v);
  }
};

// The operand whose product with x is the sum of x (ZEROS) or what the offset of the operands and the zero point 8 take off: -136
// times it (136 is a bf16 number), in all four accumulators of a lane.
template <bool ZEROS>
__device__ __forceinline__ bf16x8_t sum_operand() {
  constexpr uint32_t V = ZEROS ? 0x3F803F80u : 0xC308C308u;
  return as_bf16x8(u32x4_t{V, V, V, V});
}

// Which outputs, inputs and rows a workgroup takes.
struct Place {
  int split, tile, z, cell;
};
__device__ __forceinline__ Place place(int splits, int tiles) {
  const int tile = (int)blockIdx.x % tiles, rest = (int)blockIdx.x / tiles, z = rest / splits;
  return {rest % splits, tile, z, z * tiles + tile};
}

// output n of rows m .. m + 3
__device__ __forceinline__ void store_four(const W4Args &a, int m, int n, f32x4_t v) {
  if (n >= a.n) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (m + r < a.m) a.y[(m + r) * a.y_stride + n] = (uint16_t)pack_bf16x2(v[r], 0.f);
}

// d += a b.  The compiler may give the sum other registers than d's, and a following product that adds to it then waits for it as for
// any other result: where less than two independent products come between (NEAR), the wait is written out.
template <bool NEAR>
__device__ __forceinline__ f32x4_t mfma(f32x4_t d, bf16x8_t a, bf16x8_t b) {
  d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, d, 0, 0, 0);
  if constexpr (NEAR) asm volatile("s_nop 7" : "+v"(d));
  return d;
}

// Matrix instructions behind this stay behind it; others may move across.
__device__ __forceinline__ void products_in_order() { __builtin_amdgcn_sched_barrier(0x3F6); }

// Scales (and zero points) of a lane's output j in the groups of a block, as loaded: whole words, with those of neighbours
// where a lane's own are less (a narrower load would have to be extended, and be waited for where it is loaded).
template <int GPB, bool ZEROS>
struct Groups {
  uint32_t s[(GPB + 1) / 2];
  uint32_t z;
  __device__ __forceinline__ void load(const W4Args &a, const W4Layout &l, int64_t block, int j) {
    const int64_t at = (block * 16 + j) * GPB;
    const unsigned char *sp = a.weight + l.scales + (GPB == 1 ? at & ~(int64_t)1 : at) * 2;
    if constexpr (GPB == 4) {
      const u32x2_t v = *reinterpret_cast<const u32x2_t *>(sp);
      s[0] = v[0];
      s[1] = v[1];
    } else {
      s[0] = *reinterpret_cast<const uint32_t *>(sp);
    }
    if constexpr (ZEROS) z = *reinterpret_cast<const uint32_t *>(a.weight + l.zeros + (at & ~(int64_t)3));
  }
  __device__ __forceinline__ void here() {
#pragma unroll
    for (int i = 0; i < (GPB + 1) / 2; ++i) asm volatile("" : "+v"(s[i]));
    if constexpr (ZEROS) asm volatile("" : "+v"(z));
  }
  __device__ __forceinline__ float scale(int g, int j) const {
    if constexpr (GPB == 1) return __uint_as_float((s[0] << (j & 1 ? 0 : 16)) & 0xFFFF0000u);
    return __uint_as_float(g & 1 ? s[g >> 1] & 0xFFFF0000u : s[g >> 1] << 16);
  }
  // where the accumulators of a group begin, from the product with sum_operand
  __device__ __forceinline__ f32x4_t first(int g, int j, f32x4_t sum) const {
    if constexpr (!ZEROS) return sum;
    const float c = -(128.f + (float)((z >> (8 * ((j * GPB + g) & 3))) & 0xFFu));
    return f32x4_t{c * sum[0], c * sum[1], c * sum[2], c * sum[3]};
  }
};

// ---- slices of 16 rows: a workgroup takes up to eight blocks of 16 outputs, each on KW wavefronts, a share of the inputs each ----
// x of the workgroup's inputs lies in LDS, so that the vector memory path carries weights alone and wavefronts do not wait for each
// other behind the first barrier; a wavefront has U blocks of weights in use and U on the way.  Bound by reading the weights: 28672 x 4096 with
// zero points (62 MB) one row 14.9 us, 7 rows 16.4 to 17.8, 8 rows 18.0 (a kernel that only reads as much: 10); 6144 x 4096 6.4 us, of which 2.2 are a launch.
template <int GROUP, bool ZEROS, int KW, int U>
__global__ __launch_bounds__(1024) void w4_few_kernel(const W4Args a, const W4Layout l, int splits, int tiles, int x_row) {
  constexpr int GPB = 128 / GROUP, STEPS = GROUP / 32;  // groups of a block of inputs, matrix instructions of a group
  const int threads = blockDim.x, NW = threads / (64 * KW);  // blocks of outputs
  extern __shared__ __align__(16) unsigned char lds[];
  uint16_t *xs = reinterpret_cast<uint16_t *>(lds);  // [rows][x_row]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 15, g4 = lane >> 4;
  const Place at = place(splits, tiles);
  const int tile = at.tile, split = at.split, m0 = at.z * 16, rows = min(16, a.m - m0);
  const int64_t block = (int64_t)tile * NW + wave / KW, nb = min(block, l.n_blocks - 1);
  const int n_kb = (int)l.k_blocks, first = (int)((int64_t)n_kb * split / splits), n_mine = (int)((int64_t)n_kb * (split + 1) / splits) - first;
  const int kb0 = first + n_mine * (wave % KW) / KW, kb1 = first + n_mine * (wave % KW + 1) / KW;
  struct Blocks {
    u32x4_t w[U];
    Groups<GPB, ZEROS> g[U];
  };
  const unsigned char *wp = a.weight + nb * n_kb * 1024 + lane * 16;
  auto load = [&](int kb, Blocks &f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = max(min(kb + u, kb1 - 1), 0);  // (past the end: the last block again, not used)
      f.w[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(wp + (int64_t)k * 1024));
      f.g[u].load(a, l, nb * n_kb + k, j);
    }
  };
  // inputs [128 first, 128 (first + n_mine)) of the rows; zeros past the last.  Asked for in front of the weights, so that they do not wait for those.
  const int per_row = n_mine * 16, total = rows * per_row;
  auto x_chunk = [&](int i) __attribute__((always_inline)) {
    const int r = i / per_row, k = first * 128 + (i - r * per_row) * 8;
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (i < total && k < a.k) v = *reinterpret_cast<const u32x4_t *>(a.x + (m0 + r) * a.x_stride + k);
    return v;
  };
  auto put_x = [&](int i, u32x4_t v) __attribute__((always_inline)) {
    const int r = i / per_row;
    if (i < total) *reinterpret_cast<u32x4_t *>(xs + r * x_row + (i - r * per_row) * 8) = v;
  };
  Blocks fa, fb;
  const u32x4_t x0 = x_chunk(threadIdx.x);
  __builtin_amdgcn_sched_barrier(0);
  load(kb0, fa);
  load(kb0 + U, fb);
  __builtin_amdgcn_sched_barrier(0);
  put_x(threadIdx.x, x0);
  for (int i = threadIdx.x + threads; i < total; i += threads) put_x(i, x_chunk(i));
  __syncthreads();
  const Unpack unpack;
  const bf16x8_t summing = sum_operand<ZEROS>();
  const uint16_t *x = xs + min(j, rows - 1) * x_row + 8 * g4 - first * 128;
  f32x4_t y = {0.f, 0.f, 0.f, 0.f};
  auto compute = [&](int kb, Blocks &f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb + u >= kb1) break;  // wave-uniform
      f.g[u].here();
      bf16x8_t xv[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) xv[s] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(x + (kb + u) * 128 + 32 * s));
#pragma unroll
      for (int g = 0; g < GPB; ++g) {
        f32x4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) d = mfma<true>(d, xv[g * STEPS + s], summing);
        d = f.g[u].first(g, j, d);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) d = mfma<true>(d, xv[g * STEPS + s], unpack(f.w[u][g * STEPS + s]));
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = __builtin_fmaf(f.g[u].scale(g, j), d[r], y[r]);
      }
    }
  };
  for (int kb = kb0; kb < kb1; kb += 2 * U) {
    compute(kb, fa);
    __builtin_amdgcn_sched_barrier(0);
    load(kb + 2 * U, fa);
    __builtin_amdgcn_sched_barrier(0);
    compute(kb + U, fb);
    __builtin_amdgcn_sched_barrier(0);
    load(kb + 3 * U, fb);
    __builtin_amdgcn_sched_barrier(0);
  }
  bool mine = block < l.n_blocks;
  if constexpr (KW > 1) {  // the first wavefront of each block adds up its shares
    __syncthreads();
    f32x4_t *sums = reinterpret_cast<f32x4_t *>(lds);
    sums[threadIdx.x] = y;
    __syncthreads();
    mine = mine && wave % KW == 0;
    if (mine)
#pragma unroll
      for (int i = 1; i < KW; ++i) y += sums[threadIdx.x + 64 * i];
  }
  if (splits > 1) {
    const __amdgpu_buffer_rsrc_t rs = parts_of(a.ws);
    const unsigned part = (unsigned)((at.cell * splits * NW + wave / KW) * 64 + lane) * 16u, step = NW * 64 * 16u;
    if (mine) put_part(rs, part + split * step, y);
    if (!last_of(a.counters + at.cell, splits, reinterpret_cast<unsigned *>(lds + threads * 16))) return;
    if (mine) {
      y = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < splits; ++i) y += get_part(rs, part + i * step);
    }
  }
  if (mine) store_four(a, m0 + 4 * g4, (int)block * 16 + j, y);
}

// ---- up to 64 rows: a workgroup of two shares of the inputs, four wavefronts each, takes 16 * MB rows and 64 * NB outputs ----
// x travels to LDS as matrix operands (a wavefront's load of 1 KB is one operand of 16 rows by 32 inputs), in a ring for each share of RING
// blocks of 128 inputs that its four wavefronts read; weights go straight to registers, two blocks before they are used.  The shares keep
// two wavefronts on a SIMD, of which one computes while the other waits for LDS (half the wavefronts: 81 us for 51 at 8192 x 28672, 61 rows, on one card), and
// are added up in LDS, which two workgroups would do through memory (53 us).
// What bounds it: issuing products and vector arithmetic.  A block is 12 MB products of a wavefront (a third of them the sum of x, which takes the
// place of unpacking to signed numbers: twice the instructions), three vector instructions for each and 4 MB reads of LDS; by themselves 12
// products take a SIMD 98 ns, with 36 vector instructions and 4 reads 146.  For 8192 x 28672, 61 rows that makes 33 us (the weights from memory
// 27), to which come a launch, the first loads, waits at barriers and 4 us of joining: 50 us in groups of 128, 54 in groups of 64, 2.4 TB/s of
// weights, 0.8 PFLOP/s with the sums.  With up to 16 rows it is bound by memory: 8192 x 28672 27 to 30 us, 4.0 to 4.4 TB/s.  More than 64 rows
// repeat it for every 64: 8192 x 28672 91 us for 65 to 128 rows, 504 for 1000 (0.93 PFLOP/s).
constexpr int TILE_RING = 4, TILE_KW = 2;

__device__ __forceinline__ void x_to_lds(const void *src, unsigned char *lds) {
  __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}

template <int GROUP, bool ZEROS, int MB, int NB>
__global__ __launch_bounds__(256 * TILE_KW, 2) void w4_tile_kernel(const W4Args a, const W4Layout l, int splits, int tiles) {
  constexpr int KW = TILE_KW, GPB = 128 / GROUP, STEPS = GROUP / 32, BLK = 4 * MB * 1024;
  // (dynamic: the compiler would let every read of a ring that it knows wait for all that is on the way to it)
  extern __shared__ __align__(16) unsigned char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3, kw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), lane = threadIdx.x & 63, j = lane & 15, g4 = lane >> 4;
  const Place at = place(splits, tiles);
  const int tile = at.tile, split = at.split, m0 = at.z * 64;
  const int64_t nb0 = ((int64_t)tile * 4 + wave) * NB;
  const int n_kb = (int)l.k_blocks, begin = (int)((int64_t)n_kb * split / splits), end = (int)((int64_t)n_kb * (split + 1) / splits);
  // (all shares take as many steps: they meet at barriers)
  const int n_steps = (end - begin + KW - 1) / KW, kb0 = begin + kw * n_steps, kb1 = min(kb0 + n_steps, end);
  unsigned char *ring = lds + kw * (TILE_RING * BLK);
  const uint16_t *x[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) x[i] = a.x + min(m0 + 16 * i + j, a.m - 1) * a.x_stride + 8 * g4;  // (rows past the last repeat it)
  // wavefront w brings step w of a block (past the inputs: the last step again, under scales of zero)
  auto request = [&](int kb) __attribute__((always_inline)) {
    const int k0 = min(min(kb, end - 1) * 128 + 32 * wave, a.k - 32);
#pragma unroll
    for (int i = 0; i < MB; ++i) x_to_lds(x[i] + k0, ring + (kb % TILE_RING) * BLK + (wave * MB + i) * 1024);
  };
  const unsigned char *wp[NB];
  int64_t gp[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t nb = min(nb0 + b, l.n_blocks - 1);
    wp[b] = a.weight + nb * n_kb * 1024 + lane * 16;
    gp[b] = nb * n_kb;
  }
  struct Block {
    u32x4_t w[NB];
    Groups<GPB, ZEROS> g[NB];
  };
  auto load = [&](int kb, Block &f) __attribute__((always_inline)) {
    const int k = min(kb, end - 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f.w[b] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(wp[b] + (int64_t)k * 1024));
      f.g[b].load(a, l, gp[b] + k, j);
    }
  };
  f32x4_t y[NB][MB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < MB; ++i) y[b][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const Unpack unpack;
  const bf16x8_t summing = sum_operand<ZEROS>();
  auto compute = [&](int kb, Block &f) __attribute__((always_inline)) {
    // scales are unpacked here, and not where they are loaded (which would wait for them there)
#pragma unroll
    for (int b = 0; b < NB; ++b) f.g[b].here();
    const unsigned char *blk = ring + (kb % TILE_RING) * BLK + lane * 16;
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      bf16x8_t xv[STEPS][MB];
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < MB; ++i) xv[s][i] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(blk + ((g * STEPS + s) * MB + i) * 1024));
      f32x4_t sum[MB];
#pragma unroll
      for (int i = 0; i < MB; ++i) sum[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < MB; ++i) {
          sum[i] = mfma<(MB < 3)>(sum[i], xv[s][i], summing);
          if (NB > 2 || i == MB - 1) products_in_order();
        }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x4_t d[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) d[i] = f.g[b].first(g, j, sum[i]);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const bf16x8_t w = unpack(f.w[b][g * STEPS + s]);
#pragma unroll
          for (int i = 0; i < MB; ++i) {
            d[i] = mfma<(MB < 3)>(d[i], xv[s][i], w);
            if (NB > 2 || i == MB - 1) products_in_order();
          }
        }
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) y[b][i][r] = __builtin_fmaf(f.g[b].scale(g, j), d[i][r], y[b][i][r]);
      }
    }
  };
  // Block kb: behind the barrier its x has landed for everybody, and the slot of block kb - 1 is free for kb + 3.  What may be
  // in flight still: x of kb + 2 and weights of kb + 1, asked for behind the weights of kb.
  constexpr int IN_FLIGHT = MB + NB * (ZEROS ? 3 : 2);
  static_assert(IN_FLIGHT < 64, "the counter's range");
  auto step = [&](int kb, Block &f) __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((IN_FLIGHT & 0xF) | ((IN_FLIGHT >> 4) << 14) | 0xF70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    request(kb + TILE_RING - 1);
    if (kb < kb1) compute(kb, f);
    __builtin_amdgcn_sched_barrier(0);
    load(kb + 2, f);
    __builtin_amdgcn_sched_barrier(0);
  };
  Block fa, fb;
  static_assert(TILE_RING == 4, "three blocks of x on the way, in the order that the steps leave them");
  request(kb0);
  request(kb0 + 1);
  __builtin_amdgcn_sched_barrier(0);
  load(kb0, fa);
  __builtin_amdgcn_sched_barrier(0);
  request(kb0 + 2);
  __builtin_amdgcn_sched_barrier(0);
  load(kb0 + 1, fb);
  __builtin_amdgcn_sched_barrier(0);
  int kb = kb0;
  for (; kb + 1 < kb0 + n_steps; kb += 2) {
    step(kb, fa);
    step(kb + 1, fb);
  }
  if (kb < kb0 + n_steps) step(kb, fa);
  __builtin_amdgcn_s_waitcnt(0x0F70);  // the look-ahead has landed before the LDS is released
  {  // the first share's wavefronts add the second's
    static_assert(KW == 2 && NB * MB * 4096 <= KW * TILE_RING * BLK, "room where x was");
    __syncthreads();
    f32x4_t *sums = reinterpret_cast<f32x4_t *>(lds) + (threadIdx.x & 255);
    if (kw > 0)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < MB; ++i) sums[(b * MB + i) * 256] = y[b][i];
    __syncthreads();
    if (kw == 0)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < MB; ++i) y[b][i] += sums[(b * MB + i) * 256];
    __syncthreads();
  }
  if (NB == 2 && splits > 1) {  // (64 outputs a wavefront are never shared: parts of 64 KB take 9 us to join)
    const __amdgpu_buffer_rsrc_t rs = parts_of(a.ws);
    const unsigned step_bytes = NB * MB * 256 * 16u, part = (unsigned)(at.cell * splits) * step_bytes + (threadIdx.x & 255) * 16u;
    if (kw == 0)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < MB; ++i) put_part(rs, part + split * step_bytes + (b * MB + i) * 4096u, y[b][i]);
    if (!last_of(a.counters + at.cell, splits, reinterpret_cast<unsigned *>(lds))) return;
    if (kw > 0) return;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < MB; ++i) y[b][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < splits; ++p) {
      f32x4_t v[NB][MB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < MB; ++i) v[b][i] = get_part(rs, part + p * step_bytes + (b * MB + i) * 4096u);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < MB; ++i) y[b][i] += v[b][i];
    }
  }
  if (kw > 0) return;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < MB; ++i) store_four(a, m0 + 16 * i + 4 * g4, (int)(nb0 + b) * 16 + j, y[b][i]);
}

// products over no inputs
__global__ __launch_bounds__(256) void w4_zero_kernel(const W4Args a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)a.m * a.n) a.y[i / a.n * a.y_stride + i % a.n] = 0;
}

// One 32-bit word of a block per thread, then a scale (and zero point) per thread.
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, int64_t n, int64_t k,
                                                     int group, unsigned char *weight, const W4Layout l) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n_words = l.n_blocks * l.k_blocks * 256;
  if (i < n_words) {
    const int s = (int)(i & 3), lane = (int)(i >> 2) & 63;
    const int64_t block = i >> 8, row = block / l.k_blocks * 16 + (lane & 15), k0 = block % l.k_blocks * 128 + 32 * s + 8 * (lane >> 4);
    uint32_t v = 0;
    if (row < n && k0 < k)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint32_t two = packed[(row * k + k0) / 2 + b];
        v |= (two & 15u) << (4 * b) | (two >> 4) << (4 * b + 16);
      }
    reinterpret_cast<uint32_t *>(weight)[i] = v;
    return;
  }
  const int64_t e = i - n_words;
  if (e >= l.n_blocks * l.groups * 16) return;
  const int gpb = 128 / group;
  const int64_t block = e / gpb / 16, row = block / l.k_blocks * 16 + e / gpb % 16, g = block % l.k_blocks * gpb + e % gpb;
  const bool in = row < n && g * group < k;
  reinterpret_cast<uint16_t *>(weight + l.scales)[e] = in ? scales[row * (k / group) + g] : (uint16_t)0;
  if (zeros) weight[l.zeros + e] = in ? zeros[row * (k / group) + g] : (unsigned char)0;
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// splits of the inputs, within the workspace and the counters
int within(const W4Args &a, int want, int64_t cells, int floats_per_part) {
  if (cells > a.n_counters) return 1;
  return std::max(1, (int)std::min<int64_t>(want, (int64_t)a.ws_floats / (cells * floats_per_part)));
}

template <int GROUP, bool ZEROS, int MB, int NB>
hipError_t run_tile(const W4Args &a, const W4Layout &l, int splits, hipStream_t stream) {
  constexpr int LDS = TILE_KW * TILE_RING * 4 * MB * 1024;
  const int tiles = ceil_div(l.n_blocks, 4 * NB), z = ceil_div(a.m, 64);
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(&w4_tile_kernel<GROUP, ZEROS, MB, NB>), LDS)) return e;
  hipLaunchKernelGGL((w4_tile_kernel<GROUP, ZEROS, MB, NB>), dim3((unsigned)(tiles * splits * z)), dim3(256 * TILE_KW), LDS, stream, a, l, splits, tiles);
  return hipGetLastError();
}

// How a product is done is chosen by expected microseconds, fitted to 11 sets of rows (1 to 64), groups and zero points times 26 shapes from 256 x
// 28672 to 28672 x 4096, each in tiles and in slices of 16 rows on 1 to 8 workgroups: 0.6 % longer than the best of them on average, 11 % at
// worst (6144 x 4096, 48 rows); tiles alone 36 %.
struct Way {
  int splits = 1, blocks = 0;  // workgroups that share outputs; blocks of outputs of a workgroup (tiles: of a wavefront; 0: not possible)
  double us = 0;
};

// Slices of 16 rows on one workgroup a CU of as many blocks of outputs as it takes, up to 16 wavefronts, two to eight of them to a block: a
// start, the blocks and the slice's x, a wavefront's blocks in turn, and the join.  28672 x 8192, 4 rows 26.5 us, in workgroups of four
// blocks 30.7; 4096 x 14336, 4 rows on two workgroups 11.2, on one 12.6.
constexpr int few_wavefronts(int blocks) { return blocks <= 2 ? 8 : blocks <= 4 ? 4 : 2; }  // of a block
constexpr int FEW_LDS = 160 * 1024;
int few_x_row(const W4Layout &l, int splits) { return ceil_div(l.k_blocks, splits) * 128 + 8; }

Way few_way(const W4Args &a, const W4Layout &l) {
  const int nb = (int)l.n_blocks, kb = (int)l.k_blocks, rows = std::min(a.m, 16);
  const int64_t z = ceil_div(a.m, 16);
  Way best;
  for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
    const int per_slice = (int)(a.n_cu / (s * z));
    if (per_slice == 0 || (s > 1 && kb < 4 * s)) break;
    const int blocks = ceil_div(nb, per_slice), steps = ceil_div(kb, s);
    const int64_t cells = ceil_div(nb, std::max(blocks, 1)) * z;
    if (blocks > 8 || rows * few_x_row(l, s) * 2 > FEW_LDS) continue;
    if (s > 1 && (cells > a.n_counters || cells * s * blocks * 256 > (int64_t)a.ws_floats)) continue;
    const int wavefronts = few_wavefronts(blocks);
    const double us = 1.6 + steps * (blocks * (a.group == 32 ? 0.036 : 0.020) + rows * 0.0058) +
                      (wavefronts == 8 ? 0.17 : wavefronts == 4 ? 0.23 : 0.38) * ceil_div(steps, wavefronts) + (s > 1 ? 0.5 + 0.48 * s : 0.0);
    if (!best.blocks || us < best.us) best = {s, blocks, us};
  }
  return best;
}

// Tiles: rounds of workgroups on the chip, in each a start and its share's steps of one block, and the join, which one workgroup does.  17000 x 8192,
// 133 tiles, 61 rows on 3 workgroups in two rounds 45.7 us, on one 48.5.  Where 32 outputs a wavefront would give more workgroups than CUs it
// takes 64, which also need fewer sums of x for a product: 57344 x 8192, 61 rows 78 us for 89, 12 rows 48 for 51; 28672 x 4096, 61
// rows on fewer CUs 31.4 for 28.0.
Way tile_way(const W4Args &a, const W4Layout &l) {
  const int64_t z = ceil_div(a.m, 64), cells = ceil_div(l.n_blocks, 8) * z;
  const int kb = (int)l.k_blocks;
  const double step = (0.65 + 0.2 * std::min(4, ceil_div(a.m, 16))) * (a.group == 32 ? 1.25 : 1.0);
  if (cells > a.n_cu) return {1, 4, 2.5 + ceil_div(ceil_div(l.n_blocks, 16) * z, a.n_cu) * (2.5 + 1.6 * step * ceil_div(kb, 2))};
  Way best;
  for (int s = 1; s <= 8 && (s == 1 || kb >= 5 * s); ++s) {
    const double us = 2.5 + ceil_div(cells * s, a.n_cu) * (2.5 + step * ceil_div(ceil_div(kb, s), 2)) + (s > 1 ? 2.5 + 0.65 * s : 0.0);
    if (!best.blocks || us < best.us) best = {s, 2, us};
  }
  return best;
}

template <int GROUP, bool ZEROS, int KW, int U>
hipError_t run_few(const W4Args &a, const W4Layout &l, const Way &way, hipStream_t stream) {
  const int tiles = ceil_div(l.n_blocks, way.blocks), z = ceil_div(a.m, 16), threads = way.blocks * KW * 64, x_row = few_x_row(l, way.splits);
  const int lds = std::max(std::min(a.m, 16) * x_row * 2, threads * 16 + 16);
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(&w4_few_kernel<GROUP, ZEROS, KW, U>), FEW_LDS)) return e;
  hipLaunchKernelGGL((w4_few_kernel<GROUP, ZEROS, KW, U>), dim3((unsigned)(tiles * way.splits * z)), dim3(threads), lds, stream, a, l, way.splits, tiles, x_row);
  return hipGetLastError();
}

template <int GROUP, bool ZEROS, int MB>
hipError_t launch_tile(const W4Args &a, const W4Layout &l, const Way &way, hipStream_t stream) {
  if (way.blocks == 4) return run_tile<GROUP, ZEROS, MB, 4>(a, l, 1, stream);
  return run_tile<GROUP, ZEROS, MB, 2>(a, l, within(a, way.splits, (int64_t)ceil_div(l.n_blocks, 8) * ceil_div(a.m, 64), 2 * MB * 1024), stream);
}

template <int GROUP, bool ZEROS>
hipError_t launch_group(const W4Args &a, const W4Layout &l, hipStream_t stream) {
  const Way few = few_way(a, l), tile = tile_way(a, l);
  if (few.blocks && few.us < tile.us) {
    const int wavefronts = few_wavefronts(few.blocks);
    if (wavefronts == 8) return run_few<GROUP, ZEROS, 8, 1>(a, l, few, stream);
    if (wavefronts == 4) return run_few<GROUP, ZEROS, 4, 2>(a, l, few, stream);
    return run_few<GROUP, ZEROS, 2, 2>(a, l, few, stream);
  }
  if (a.m <= 16) return launch_tile<GROUP, ZEROS, 1>(a, l, tile, stream);
  if (a.m <= 32) return launch_tile<GROUP, ZEROS, 2>(a, l, tile, stream);
  if (a.m <= 48) return launch_tile<GROUP, ZEROS, 3>(a, l, tile, stream);
  return launch_tile<GROUP, ZEROS, 4>(a, l, tile, stream);
}

template <int GROUP>
hipError_t launch_zeros(const W4Args &a, const W4Layout &l, hipStream_t stream) {
  return a.with_zeros ? launch_group<GROUP, true>(a, l, stream) : launch_group<GROUP, false>(a, l, stream);
}

}  // namespace

hipError_t launch_w4_linear(const W4Args &a, hipStream_t stream) {
  if (a.m <= 0 || a.n <= 0) return hipSuccess;
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.with_zeros);
  if (a.k == 0) {
    hipLaunchKernelGGL(w4_zero_kernel, dim3((unsigned)(((int64_t)a.m * a.n + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
  }
  if (a.group == 32) return launch_zeros<32>(a, l, stream);
  if (a.group == 64) return launch_zeros<64>(a, l, stream);
  if (a.group == 128) return launch_zeros<128>(a, l, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_w4_pack(const uint8_t *packed, const uint16_t *scales, const uint8_t *zeros, int64_t n, int64_t k, int group,
                          unsigned char *weight, hipStream_t stream) {
  const W4Layout l = w4_layout(n, k, group, zeros != nullptr);
  const int64_t threads = l.n_blocks * l.k_blocks * 256 + l.n_blocks * l.groups * 16;
  if (threads <= 0) return hipSuccess;
  hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, packed, scales, zeros, n, k, group, weight, l);
  return hipGetLastError();
}

}  // namespace bs

namespace {

constexpr int64_t MOST = 1 << 24;  // outputs, inputs and rows of a product: grids and byte offsets stay far inside their types

bool shape_ok(int64_t n, int64_t k, int32_t group) {
  return n >= 0 && k >= 0 && n <= MOST && k <= MOST && (group == 32 || group == 64 || group == 128) && k % group == 0 &&
         (n + 15) / 16 * ((k + 127) / 128) <= (int64_t)1 << 30;
}

}  // namespace

extern "C" {

int64_t bs_w4_bytes(int64_t n, int64_t k, int32_t group, int32_t with_zeros) {
  return shape_ok(n, k, group) ? w4_layout(n, k, group, with_zeros != 0).bytes : 0;
}

int bs_w4_pack(bs_ctx *c, const void *packed, const void *scales, const void *zeros, int64_t n, int64_t k, int32_t group, void *weight,
               void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    const CtxView v = ctx_view(c);
    if (v.device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
    if (!shape_ok(n, k, group)) return ctx_fail(c, BS_EUNSUPPORTED, "bs_w4_pack: n=%lld k=%lld group=%d (group 32, 64 or 128 and a divisor of k)", (long long)n, (long long)k, group);
    if (n == 0 || k == 0) return BS_OK;
    if (!packed || !scales || !weight) return ctx_fail(c, BS_EINVAL, "bs_w4_pack: NULL pointer");
    if (reinterpret_cast<uintptr_t>(weight) & 15) return ctx_fail(c, BS_EINVAL, "bs_w4_pack: the weight must be 16-byte aligned");
    CTX_HIP_TRY(c, hipSetDevice(v.device));
    CTX_HIP_TRY(c, launch_w4_pack((const uint8_t *)packed, (const uint16_t *)scales, (const uint8_t *)zeros, n, k, group, (unsigned char *)weight,
                                  (hipStream_t)stream));
    return BS_OK;
  });
}

int bs_w4_linear(bs_ctx *c, const void *x, int64_t x_stride, const void *weight, int64_t m, int64_t n, int64_t k, int32_t group,
                 int32_t with_zeros, void *y, int64_t y_stride, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    const CtxView v = ctx_view(c);
    if (v.device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
    if (!shape_ok(n, k, group) || m < 0 || m > 65535 * 64)
      return ctx_fail(c, BS_EUNSUPPORTED, "bs_w4_linear: m=%lld n=%lld k=%lld group=%d (group 32, 64 or 128 and a divisor of k)", (long long)m, (long long)n, (long long)k, group);
    if (m == 0 || n == 0) return BS_OK;
    if (!y || (k > 0 && (!x || !weight))) return ctx_fail(c, BS_EINVAL, "bs_w4_linear: NULL pointer");
    if (x_stride < k || x_stride % 8 || y_stride < n || (reinterpret_cast<uintptr_t>(x) & 15) || (reinterpret_cast<uintptr_t>(weight) & 15))
      return ctx_fail(c, BS_EINVAL, "bs_w4_linear: strides %lld and %lld of rows of %lld and %lld elements (x and the weight 16-byte aligned, x's stride a multiple of 8)",
                      (long long)x_stride, (long long)y_stride, (long long)k, (long long)n);
    CTX_HIP_TRY(c, hipSetDevice(v.device));
    W4Args a{};
    a.x = (const uint16_t *)x; a.weight = (const unsigned char *)weight; a.y = (uint16_t *)y;
    a.x_stride = x_stride; a.y_stride = y_stride;
    a.m = (int)m; a.n = (int)n; a.k = (int)k; a.group = group; a.with_zeros = with_zeros != 0;
    a.ws = v.ws; a.counters = v.counters; a.ws_floats = v.ws_floats; a.n_counters = v.n_counters; a.n_cu = v.n_cu;
    CTX_HIP_TRY(c, launch_w4_linear(a, (hipStream_t)stream));
    return BS_OK;
  });
}

}  // extern "C"
