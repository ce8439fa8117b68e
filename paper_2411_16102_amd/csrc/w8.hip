// Products of 8-bit integers with a scale for each row of either operand, and the rows' way there.
//
// y[m, n] = row_scale[m] col_scale[n] sum over k of xq[m, k] w[n, k]: sums of integers in 32 bits, exact whatever their order, then two products in
// 32 bits (within their range where the result is: see W8RowScale) and one rounding.  v_mfma_i32_16x16x64_i8 takes the same 16 bytes of a row from a lane as the bf16 instruction of half the
// length, and as long, so tiles and rings are those of gemm.hip with rows of k / 2 numbers: twice the operations for every byte that moves.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/blendstep_bits.h"
#include "context.hpp"
#include "gemm.hpp"
#include "attn_device.hpp"

namespace bs {
namespace {
__device__ __align__(16) uint16_t g_gemm_zero_chunk[8];
}
}  // namespace bs

#include "gemm_device.hpp"

namespace bs {
namespace {

// ------------------------------------------------------------------------------
// rows as 8-bit integers
// ------------------------------------------------------------------------------
// scale = greatest magnitude / 127, q = x / scale to the nearest integer, quotients rounded to 32 bits (by the residual, which is exact) so that the result
// does not depend on how they are computed.  A workgroup of T threads per row, eight numbers a thread at a time; the first KEPT times eight
// stay in registers between the two passes, what is behind them is read again.
constexpr int QUANT_KEPT = 4;
constexpr float LEAST = 7.8886090522101181e-31f;  // 2^-100: of a row's greatest magnitude, so that scales and their inverses are ordinary numbers

struct QuantArgs {
  const uint16_t *x;
  int64_t x_stride;
  int8_t *q;
  float *scale;
  int m, k;
};

struct RowScale {
  float scale, inverse;
  bool bad;  // a NaN or an infinity: the row's results are NaN
  __device__ __forceinline__ explicit RowScale(uint32_t most) {  // bits of the greatest magnitude
    bad = most >= 0x7F80u;
    scale = bad ? __builtin_nanf("") : fmaxf(__uint_as_float(most << 16), LEAST) / 127.f;
    inverse = 1.f / scale;
  }
  __device__ __forceinline__ u32x2_t integers(u32x4_t v) const {
#pragma clang fp contract(off)
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16);
      float c = f * inverse;
      c = __builtin_fmaf(__builtin_fmaf(-c, scale, f), inverse, c);
      const int n = bad ? 0 : (int)__builtin_amdgcn_fmed3f(__builtin_rintf(c), -127.f, 127.f);
      w[i >> 2] |= (uint32_t)(n & 255) << (8 * (i & 3));
    }
    return u32x2_t{w[0], w[1]};
  }
};

template <int T>
__global__ __launch_bounds__(T) void w8_quantize_kernel(const QuantArgs a) {
  const int64_t row = blockIdx.x;
  const uint16_t *x = a.x + row * a.x_stride;
  u32x4_t kept[QUANT_KEPT];
  uint32_t most = 0;
  auto look = [&](u32x4_t v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, max(v[i] & 0x7FFFu, v[i] >> 16 & 0x7FFFu));
  };
#pragma unroll
  for (int i = 0; i < QUANT_KEPT; ++i) {
    const int at = (i * T + (int)threadIdx.x) * 8;
    kept[i] = at < a.k ? attn_dev::ld16(x + at) : u32x4_t{0u, 0u, 0u, 0u};
  }
#pragma unroll
  for (int i = 0; i < QUANT_KEPT; ++i) look(kept[i]);
#pragma unroll 4
  for (int at = (QUANT_KEPT * T + (int)threadIdx.x) * 8; at < a.k; at += T * 8) look(attn_dev::ld16(x + at));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
  if constexpr (T > 64) {
    __shared__ uint32_t part[T / 64];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T / 64; ++i) most = max(most, part[i]);
  }
  const RowScale scale(most);
  if (threadIdx.x == 0) a.scale[row] = scale.scale;
  int8_t *q = a.q + row * a.k;
  auto put = [&](u32x4_t v, int at) { *reinterpret_cast<u32x2_t *>(q + at) = scale.integers(v); };
#pragma unroll
  for (int i = 0; i < QUANT_KEPT; ++i) {
    const int at = (i * T + (int)threadIdx.x) * 8;
    if (at < a.k) put(kept[i], at);
  }
#pragma unroll 4
  for (int at = (QUANT_KEPT * T + (int)threadIdx.x) * 8; at < a.k; at += T * 8) put(attn_dev::ld16(x + at), at);
}

constexpr int MOST_LAUNCH = 1 << 30, FEW_LONG_ROWS = 256;  // threads; rows of more than 8192 inputs
hipError_t launch_quantize(const QuantArgs &a, hipStream_t stream) {
  if (a.m <= 0) return hipSuccess;
  // About sixteen numbers a thread; of few long rows more threads ask at once.  (us with 64, 128, 256, 512 threads: 3000 rows of 1024 4.7, 5.1, 6.1, 9.0;
  // 2560 of 4096 9.8, 9.2, 8.9, 10.4; 4000 of 14336 47, 42, 38, 30.  33 rows of 28672: 10.3 with 256, 5.2 with 1024;
  // 120 and 600 rows of 14336: with 512 and 1024 alike, and 8.4 and 9.1.)
  const auto rows_of = [&](auto threads) -> hipError_t {
    for (int m0 = 0; m0 < a.m; m0 += MOST_LAUNCH / threads()) {  // (a launch has less than 2^32 threads)
      QuantArgs part = a;
      part.x += (int64_t)m0 * a.x_stride;
      part.q += (int64_t)m0 * a.k;
      part.scale += m0;
      part.m = std::min(MOST_LAUNCH / threads(), a.m - m0);
      hipLaunchKernelGGL((w8_quantize_kernel<threads()>), dim3(part.m), dim3(threads()), 0, stream, part);
      if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
  };
  if (a.k <= 1024) return rows_of(std::integral_constant<int, 64>{});
  if (a.k <= 2048) return rows_of(std::integral_constant<int, 128>{});
  if (a.k <= 8192) return rows_of(std::integral_constant<int, 256>{});
  return a.m <= FEW_LONG_ROWS ? rows_of(std::integral_constant<int, 1024>{}) : rows_of(std::integral_constant<int, 512>{});
}

// ------------------------------------------------------------------------------
// products
// ------------------------------------------------------------------------------
// adds the k_splits sums of four results and scales them
__global__ __launch_bounds__(256) void w8_reduce_kernel(const GemmArgs a) {
  const int stride = w8_part_stride(a.N), quads = stride / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.M * quads) return;
  const int m = (int)(i / quads), n = (int)(i % quads) * 4;
  const i32x4_t *p = reinterpret_cast<const i32x4_t *>(reinterpret_cast<const int32_t *>(a.sk_ws) + (size_t)m * stride + n);
  const size_t plane = (size_t)a.M * stride / 4;
  i32x4_t s = {0, 0, 0, 0};
#pragma unroll 8
  for (int k = 0; k < a.k_splits; ++k) s += p[k * plane];
  const W8RowScale by(a.row_scale[m]);
  f32x4_t v = w8_sums(s) * by.scale;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= a.col_scale[min(n + e, a.N - 1)];
  store_scaled4(a.C + (size_t)m * a.ldc + n, v * by.back, n, a.N, ((reinterpret_cast<uintptr_t>(a.C) | (uintptr_t)a.ldc * 2) & 7) == 0);
}

// Up to four rows: rows as integers and their product in one launch.  As gemm_rows_kernel, but that the rows, brought over as they are and first,
// become integers in LDS behind the first requests for weights; rings hold weights alone.  (The greatest magnitudes are exchanged through `part`, and before it reads
// that the compiler waits for every request, as one that may write there: the first weights have landed when integers are made, and k-tiles that the ring has no
// room for are a second round trip.  One row of 4096 by 6144 outputs, four k-tiles a wavefront and room for three: 8.0 us, a launch and reads 6.4.)
constexpr int FEW_M = 4, FEW_RED = 8 * 1024;  // rows; bytes of the sums
constexpr int FEW_LDS(int ni, int s, int kb) { return 8 * s * ni * 2048 + FEW_RED + kb * 1536 + 256; }  // (reads of the last k-tile may pass the integers' end)
struct FewArgs {
  GemmArgs g;  // without A
  const uint16_t *x;
  int64_t x_stride;
};
template <int NI, int S, int KB>  // blocks of 16 outputs, k-tiles of a ring, KB of rows as they come
__global__ __launch_bounds__(512) void w8_few_kernel(const FewArgs f, const int n_items) {
  constexpr int L = 2 * NI, STAGE = L * 1024;
  static_assert(S >= 2 && FEW_LDS(NI, S, KB) + 64 <= LDS_CU && S * L < 64, "the rings, and the vmcnt field");
  extern __shared__ __align__(16) unsigned char smem[];
  const GemmArgs &a = f.g;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  unsigned char *ring = smem + wave * S * STAGE;
  i32x4_t *red = reinterpret_cast<i32x4_t *>(smem + 8 * S * STAGE);  // [8][64]
  unsigned char *raw = smem + 8 * S * STAGE + FEW_RED, *ints = raw + KB * 1024;
  __shared__ uint32_t part[8];
  const int k = 2 * a.K;
  auto dma = [](const void *p, unsigned char *lds) {
    __builtin_amdgcn_global_load_lds(p, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
  };
  // the rows, one behind the other, 1 KB a request
  const int chunks = a.M * (k / 8);
  for (int c = wave * 64; c < chunks; c += 512) {
    const int i = min(c + lane, chunks - 1);
    dma(f.x + (int64_t)(i / (k / 8)) * f.x_stride + i % (k / 8) * 8, raw + c * 16);
  }
  // requests: 8 lanes per row of 128 bytes, chunks swizzled as in gemm_tile
  const int g_row = lane >> 3, g_slot = lane & 7;
  const int chunk[2] = {g_slot ^ (g_row >> 1), g_slot ^ ((g_row + 8) >> 1)};  // rows g_row and g_row + 8 of a block
  uint32_t off_w[L];
  auto set_item = [&](int item) {
#pragma unroll
    for (int i = 0; i < L; ++i) off_w[i] = (uint32_t)(((size_t)min(item * NI * 16 + i * 8 + g_row, a.N - 1) * a.ldb + chunk[i & 1] * 8) * 2);
  };
  const int nk = (a.K + BK - 1) / BK;
  const int n = nk > wave ? (nk - wave + 7) / 8 : 0;  // k-tiles of this wavefront per item
  const int mine = (n_items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
  const int total = n * mine;
  int i_item = (int)blockIdx.x, i_k = 0, i_slot = 0, issued = 0;
  auto issue = [&]() __attribute__((always_inline)) {
    const int kt = wave + 8 * i_k;
    const unsigned char *bw = reinterpret_cast<const unsigned char *>(a.B) + (size_t)kt * 128;
    unsigned char *dst = ring + i_slot * STAGE;
    const int beyond = (kt + 1) * BK > a.K ? a.K - kt * BK : BK;  // first number of the k-tile that lies beyond K
#pragma unroll
    for (int i = 0; i < L; ++i) dma(chunk[i & 1] * 8 >= beyond ? (const void *)g_gemm_zero_chunk : bw + off_w[i], dst + i * 1024);
    ++issued;
    i_slot = i_slot + 1 == S ? 0 : i_slot + 1;
    if (++i_k == n) {
      i_k = 0;
      i_item += (int)gridDim.x;
      if (i_item < n_items) set_item(i_item);
    }
  };
  if (total > 0) set_item(i_item);
  for (int s = 0; s < S && issued < total; ++s) issue();
  wait_for_all_but<L>(issued, std::make_integer_sequence<int, S + 1>{});  // the rows have landed
  __builtin_amdgcn_s_barrier();
  // 512 / rows threads a row (as a power of two), the greatest magnitude of it among their wavefronts
  const int shift = a.M > 2 ? 7 : a.M > 1 ? 8 : 9, row = t >> shift, at0 = (t & ((1 << shift) - 1)) * 8, step = 8 << shift;
  const u32x4_t *mine_raw = reinterpret_cast<const u32x4_t *>(raw + (size_t)min(row, a.M - 1) * k * 2);
  uint32_t most = 0;
  for (int at = at0; at < k; at += step) {
    const u32x4_t v = mine_raw[at / 8];
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, max(v[i] & 0x7FFFu, v[i] >> 16 & 0x7FFFu));
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
  if (lane == 0) part[wave] = most;
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));
  __builtin_amdgcn_s_barrier();
  const auto scale_of = [&](int r) {
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = (i * 64) >> shift == r ? max(v, part[i]) : v;
    return RowScale(v);
  };
  if (row < a.M) {
    const RowScale scale = scale_of(row);
    for (int at = at0; at < k; at += step) *reinterpret_cast<u32x2_t *>(ints + row * k + at) = scale.integers(mine_raw[at / 8]);
  }
  const W8RowScale by(scale_of(min(lr, a.M - 1)).scale);
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));
  __builtin_amdgcn_s_barrier();

  const int sw = (lr >> 1) & 7;
  const unsigned char *x_row = ints + min(lr, a.M - 1) * k;
  int slot = 0, left = total, turn = 0;
  for (int item = (int)blockIdx.x; item < n_items; item += (int)gridDim.x, ++turn) {
    i32x4_t acc[NI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) acc[ni] = i32x4_t{0, 0, 0, 0};
    for (int i = 0; i < n; ++i) {
      --left;  // k-tiles behind this one
      if (left >= S - 1) {
        __builtin_amdgcn_s_waitcnt(waitcnt_imm((S - 1) * L, false));
      } else {
        wait_for_all_but<L>(left, std::make_integer_sequence<int, S - 1>{});
      }
      const unsigned char *st = ring + slot * STAGE, *xs = x_row + (wave + 8 * i) * 128;
      bf16x8_t w[2][NI], x[2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int ch = ((ks * 4 + lg) ^ sw) << 4;
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) w[ks][ni] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(st + ni * 2048 + lr * 128 + ch));
        x[ks] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(xs + (ks * 4 + lg) * 16));
      }
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));  // the slot may be filled again
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) gemm_mfma(acc[ni], w[ks][ni], x[ks]);
      if (left >= S) issue();
      slot = slot + 1 == S ? 0 : slot + 1;
    }
    // the partial sums of 16 weight rows at a time meet; the requests in flight are left alone
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));
      __builtin_amdgcn_s_barrier();  // nobody reads the sums before these any more
      red[wave * 64 + lane] = acc[ni];
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));
      __builtin_amdgcn_s_barrier();
      const int n0 = (item * NI + ni) * 16 + 4 * lg;
      if (wave != (turn * NI + ni) % 8 || lr >= a.M || n0 >= a.N) continue;
      i32x4_t sum = red[lane];
#pragma unroll
      for (int v = 1; v < 8; ++v) sum += red[v * 64 + lane];
      f32x4_t v = __builtin_convertvector(sum, f32x4_t) * by.scale;  // (rows within -127 .. 127: every sum stays in 32 bits)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= a.col_scale[min(n0 + e, a.N - 1)];
      store_scaled4(a.C + (size_t)lr * a.ldc + n0, v * by.back, n0, a.N, ((reinterpret_cast<uintptr_t>(a.C) | (uintptr_t)a.ldc * 2) & 7) == 0);
    }
  }
}

template <int NI, int S, int KB>
hipError_t launch_few(const FewArgs &f, hipStream_t stream) {
  const int64_t items = (rows_blocks(f.g.N, EPI_W8) + NI - 1) / NI, rounds = (items + f.g.n_cu - 1) / f.g.n_cu;
  if (f.g.M > FEW_M || (int64_t)f.g.M * f.g.K * 4 > KB * 1024) return hipErrorInvalidValue;
  auto kern = w8_few_kernel<NI, S, KB>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), FEW_LDS(NI, S, KB))) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((items + rounds - 1) / rounds)), dim3(512), FEW_LDS(NI, S, KB), stream, f, (int)items);
  return hipGetLastError();
}

// Whether rows go through it, and with how many blocks of outputs.
constexpr int FEW_KB = 56;
bool few_rows(int64_t m, int64_t k) { return m <= FEW_M && 2 * m * k <= FEW_KB * 1024; }
hipError_t launch_few_rows(const FewArgs &f, int ni, hipStream_t stream) {
  const bool small = (int64_t)f.g.M * f.g.K * 4 <= 16 * 1024;
  if (ni == 1) return small ? launch_few<1, 7, 16>(f, stream) : launch_few<1, 4, FEW_KB>(f, stream);
  return small ? launch_few<2, 3, 16>(f, stream) : launch_few<2, 2, FEW_KB>(f, stream);
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DEEP>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, 2) void w8_tile_kernel(const GemmArgs a) {
  gemm_tile<BM, BN, WAVES_M, WAVES_N, EPI, 64, DEEP>(a, (int)blockIdx.x);
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DEEP>
hipError_t launch_tiles(const GemmArgs &a, hipStream_t stream) {
  constexpr int LDS = DEEP ? LDS_CU : ring_bytes(WAVES_M * WAVES_N);
  auto kern = w8_tile_kernel<BM, BN, WAVES_M, WAVES_N, EPI, DEEP>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), LDS)) return e;
  const int64_t tiles = (int64_t)((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN) * a.k_splits;
  if (tiles > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(WAVES_M * WAVES_N * 64), LDS, stream, a);
  return hipGetLastError();
}

template <int MI, int NI>
hipError_t launch_rows(const GemmArgs &a, hipStream_t stream) {
  typedef RowsKernel<MI, NI> R;
  const int tiles_m = (a.M + 16 * MI - 1) / (16 * MI);
  if (tiles_m * 16 * MI > ROWS_MAX_M) return hipErrorInvalidValue;
  const int64_t items = (int64_t)tiles_m * ((rows_blocks(a.N, EPI_W8) + NI - 1) / NI), rounds = (items + a.n_cu - 1) / a.n_cu;
  if (items >= (1L << 30)) return hipErrorInvalidValue;
  auto kern = gemm_rows_kernel<MI, NI, true>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), R::LDS)) return e;
  // as many workgroups as give each the same number of items
  hipLaunchKernelGGL(kern, dim3((unsigned)((items + rounds - 1) / rounds)), dim3(512), R::LDS, stream, a, (int)EPI_W8, 64, tiles_m, (int)items);
  return hipGetLastError();
}

enum Shape { ROWS_11, ROWS_12, ROWS_21, ROWS_22, D64, SMALL, SLIM, WIDE, TALL, MID, BIG, N_SHAPES };
struct Plan {
  int shape, splits;
};

template <int EPI>
hipError_t launch_shape(int shape, const GemmArgs &a, hipStream_t stream) {
  switch (shape) {
    case D64: return launch_tiles<64, 128, 4, 2, EPI, 2>(a, stream);
    case SMALL: return launch_tiles<128, 128, 2, 2, EPI, 0>(a, stream);
    case SLIM: return launch_tiles<192, 128, 4, 2, EPI, 0>(a, stream);
    case WIDE: return launch_tiles<128, 256, 2, 4, EPI, 0>(a, stream);
    case TALL: return launch_tiles<160, 256, 2, 4, EPI, 0>(a, stream);
    case MID: return launch_tiles<192, 256, 2, 4, EPI, 0>(a, stream);
    case BIG: return launch_tiles<256, 256, 2, 4, EPI, 0>(a, stream);
  }
  return hipErrorInvalidValue;
}

// Expected microseconds of a product, by which its shape and its ranges of k are chosen: a launch, rounds of workgroups that take some time each
// and for every 128 inputs (the last round, of a chip that is filled in part, less), or its bytes, and the second kernel of ranges.  Fitted to
// 11 000 products (1 to 5000 rows, 256 to 28672 outputs, 1024 to 28672 inputs, weights cold) timed in every shape and range: the choice is 1.8 % off the best
// on average, 10 % for one in twenty, 37 % at worst (29 rows, 17736 outputs, 14656 inputs: 82 us, 60 on tiles of 128 rows cut three ways).
// SLIM came later: of 3000 products of 100 to 5000 rows it is chosen for 350, and the choice 1.7 % off the best, 2.6 without it
// (1093 rows, 4096 x 4096: 192 of its tiles 25.6 us; 144 of WIDE's 31.2, 288 of SMALL's, of which 32 CUs have two, 30.9).
struct Cost {
  int rows, outputs, per_cu;          // of a workgroup; workgroups that a CU takes at once
  double launch, round, tile, full;   // tile: of 128 inputs on an idle chip; full: more on a full one
  double per_mb;                      // of the operands
  double second, second_per_mb;       // the kernel behind ranges, and its bytes
};
constexpr Cost COSTS[N_SHAPES] = {
    {16, 16, 1, 4.112, 0.383, 0.034, 0.048, 0.162, 0, 0},
    {16, 32, 1, 3.917, 0.417, 0.066, 0.099, 0.168, 0, 0},
    {32, 16, 1, 3.96, 0.369, 0.051, 0.043, 0.181, 0, 0},
    {32, 32, 1, 3.431, 0.817, 0.083, 0.089, 0.171, 0, 0},
    {64, 128, 1, 0.476, 5.102, 0.319, 0.32, 0.179, 3.623, 0.236},
    {128, 128, 2, 3.935, 2.699, 0.929, 0.067, 0.212, 3.112, 0.339},
    {192, 128, 1, 2.62, 3.553, 0.582, 0.131, 0.255, 3.027, 0.383},
    {128, 256, 1, 3.991, 2.628, 0.767, 0.13, 0.211, 3.069, 0.341},
    {160, 256, 1, 3.97, 3.739, 0.832, 0.168, 0.226, 2.774, 0.313},
    {192, 256, 1, 4.568, 3.834, 0.895, 0.231, 0.232, 2.284, 0.304},
    {256, 256, 1, 4.977, 5.622, 1.018, 0.349, 0.25, 1.588, 0.282},
};
constexpr double HALF_ROUND = 1.572, HALF_TILE = 0.505, HALF_FULL = 0.113;  // SMALL, a last round that leaves a CU one of its two workgroups

double expected_us(int shape, int splits, int64_t m, int64_t n, int64_t k, int n_cu) {
  const Cost &c = COSTS[shape];
  const int64_t wgs = (m + c.rows - 1) / c.rows * ((n + c.outputs - 1) / c.outputs) * splits, slots = (int64_t)n_cu * c.per_cu;
  const double tiles = (double)((k + 127) / 128) / splits, last = (double)(wgs % slots) / (double)slots;
  double us = c.launch + (double)(wgs / slots) * (c.round + tiles * (c.tile + c.full));
  if (last > 0.0) us += c.per_cu == 2 && last <= 0.5 ? HALF_ROUND + tiles * (HALF_TILE + HALF_FULL * 2.0 * last) : c.round + tiles * (c.tile + c.full * last);
  us = std::max(us, c.launch + 1e-6 * (double)(n * k + 2 * m * n + m * k) * c.per_mb);
  return splits == 1 ? us : us + c.second + c.second_per_mb * 4e-6 * (double)splits * (double)m * (double)n;
}

Plan plan_of(int64_t m, int64_t n, int64_t k, int n_cu, size_t ws_floats) {
  Plan best = {BIG, 1};
  double least = 1e300;
  for (int shape = 0; shape < N_SHAPES; ++shape) {
    const Cost &c = COSTS[shape];
    if (shape < D64) {
      // (weight rows 8 KB apart in pairs of blocks: every workgroup asks few memory channels at a time, 14336 x 8192 27.6 us against 21.6)
      if (m > (c.rows == 16 ? 16 : 64) || (c.outputs == 32 && k % 8192 == 0)) continue;
    } else if (shape == D64 ? m > 128 : c.rows >= 2 * m && shape != SMALL) {
      continue;
    }
    for (int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
      const int64_t tiles = (m + c.rows - 1) / c.rows * ((n + c.outputs - 1) / c.outputs);
      if (splits > 1 && (shape < D64 || tiles * splits > 900 || k < 512 * splits || (size_t)(splits * m * w8_part_stride((int)n)) > ws_floats)) break;
      const double us = expected_us(shape, splits, m, n, k, n_cu);
      if (us < least) {
        least = us;
        best = {shape, splits};
      }
    }
  }
  return best;
}

int few_blocks(int64_t n, int64_t k, int n_cu) {
  return k % 8192 != 0 && expected_us(ROWS_12, 1, 1, n, k, n_cu) < expected_us(ROWS_11, 1, 1, n, k, n_cu) ? 2 : 1;
}

hipError_t launch_product(GemmArgs a, size_t ws_floats, hipStream_t stream) {
  Plan p = plan_of(a.M, a.N, 2 * (int64_t)a.K, a.n_cu, ws_floats);
  a.k_splits = p.splits;
  switch (p.shape) {
    case ROWS_11: return launch_rows<1, 1>(a, stream);
    case ROWS_12: return launch_rows<1, 2>(a, stream);
    case ROWS_21: return launch_rows<2, 1>(a, stream);
    case ROWS_22: return launch_rows<2, 2>(a, stream);
  }
  if (p.splits == 1) return launch_shape<EPI_W8>(p.shape, a, stream);
  if (const hipError_t e = launch_shape<EPI_W8_PARTIAL>(p.shape, a, stream)) return e;
  const int64_t quads = (int64_t)a.M * (w8_part_stride(a.N) / 4);
  hipLaunchKernelGGL(w8_reduce_kernel, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

constexpr int64_t MOST_BYTES = 0xFFFF0000;  // of an operand that a launch sees (offsets are 32 bits)
constexpr int64_t MOST_K = 131072;          // 128 * 128 k stays in 32 bits, but for one sum (see w8_sums)
constexpr int64_t MOST_ROWS = 1 << 30;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int check_product(bs_ctx *c, const char *what, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, const void *y, int64_t y_stride) {
  if (ctx_view(c).device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
  if (m < 0 || m > MOST_ROWS || n < 0 || n > MOST_ROWS || k < 16 || k % 16 || k > MOST_K || y_stride > 0x7fffffff)
    return ctx_fail(c, BS_EUNSUPPORTED, "%s: m=%lld n=%lld k=%lld (k a multiple of 16 up to %lld), rows of y %lld apart", what, (long long)m, (long long)n, (long long)k,
                    (long long)MOST_K, (long long)y_stride);
  if (m == 0 || n == 0) return BS_OK;
  if (!weight || !weight_scales || !y) return ctx_fail(c, BS_EINVAL, "%s: NULL pointer", what);
  if (y_stride < n || !aligned16(weight)) return ctx_fail(c, BS_EINVAL, "%s: rows of %lld elements at a stride of %lld (the weight 16-byte aligned)", what, (long long)n, (long long)y_stride);
  return BS_OK;
}

GemmArgs product_args(bs_ctx *c, const int8_t *q, const float *scales, const void *weight, const float *weight_scales, int m, int n, int64_t k, void *y,
                      int64_t y_stride) {
  const CtxView v = ctx_view(c);
  GemmArgs a{};
  a.A = (const uint16_t *)q;
  a.B = (const uint16_t *)weight;
  a.M = m;
  a.N = n;
  a.K = a.lda = a.ldb = (int)(k / 2);
  a.n_cu = v.n_cu;
  a.C = (uint16_t *)y;
  a.ldc = (int)y_stride;
  a.row_scale = scales;
  a.col_scale = weight_scales;
  a.sk_ws = v.ws;
  return a;
}

int products(bs_ctx *c, const int8_t *q, const float *scales, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, void *y,
             int64_t y_stride, hipStream_t stream) {
  CTX_HIP_TRY(c, hipSetDevice(ctx_view(c).device));
  // ranges of rows and of outputs whose operands offsets of 32 bits reach
  const int64_t most = MOST_BYTES / k / 256 * 256;
  for (int64_t m0 = 0; m0 < m; m0 += most)
    for (int64_t n0 = 0; n0 < n; n0 += most) {
      const GemmArgs a = product_args(c, q + m0 * k, scales + m0, (const int8_t *)weight + n0 * k, weight_scales + n0, (int)std::min(most, m - m0), (int)std::min(most, n - n0), k,
                                      (uint16_t *)y + m0 * y_stride + n0, y_stride);
      CTX_HIP_TRY(c, launch_product(a, ctx_view(c).ws_floats, stream));
    }
  return BS_OK;
}

}  // namespace
}  // namespace bs

using namespace bs;

extern "C" {

int bs_w8_quantize(bs_ctx *c, const void *x, int64_t x_stride, int64_t m, int64_t k, void *q, float *scales, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    const CtxView v = ctx_view(c);
    if (v.device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
    if (m < 0 || m > MOST_ROWS || k < 16 || k % 16 || k > MOST_K)
      return ctx_fail(c, BS_EUNSUPPORTED, "bs_w8_quantize: m=%lld k=%lld (k a multiple of 16 up to %lld)", (long long)m, (long long)k, (long long)MOST_K);
    if (m == 0) return BS_OK;
    if (!x || !q || !scales) return ctx_fail(c, BS_EINVAL, "bs_w8_quantize: NULL pointer");
    if (x_stride < k || x_stride % 8 || !aligned16(x) || !aligned16(q))
      return ctx_fail(c, BS_EINVAL, "bs_w8_quantize: rows of %lld elements at a stride of %lld (16-byte aligned, the stride a multiple of 8)", (long long)k, (long long)x_stride);
    CTX_HIP_TRY(c, hipSetDevice(v.device));
    QuantArgs a{};
    a.x = (const uint16_t *)x;
    a.x_stride = x_stride;
    a.q = (int8_t *)q;
    a.scale = scales;
    a.m = (int)m;
    a.k = (int)k;
    CTX_HIP_TRY(c, launch_quantize(a, (hipStream_t)stream));
    return BS_OK;
  });
}

int bs_w8_division(bs_ctx *c, int64_t m, int64_t n, int64_t k, int32_t *rows, int32_t *outputs, int32_t *ranges) {
  if (!c) return BS_EINVAL;
  if (m < 1 || m > MOST_ROWS || n < 1 || n > MOST_ROWS || k < 16 || k % 16 || k > MOST_K || !rows || !outputs || !ranges)
    return ctx_fail(c, BS_EINVAL, "bs_w8_division: m=%lld n=%lld k=%lld", (long long)m, (long long)n, (long long)k);
  const CtxView v = ctx_view(c);
  const Plan p = plan_of(m, n, k, v.n_cu, gemm_sk_workspace_floats());
  *rows = COSTS[p.shape].rows;
  *outputs = COSTS[p.shape].outputs;
  *ranges = p.splits;
  return BS_OK;
}

int64_t bs_w8_scratch_bytes(int64_t m, int64_t k) {
  if (m <= 0 || k <= 0 || few_rows(m, k)) return 0;
  return (4 * m + 15) / 16 * 16 + m * k;
}

int bs_w8_linear(bs_ctx *c, const void *q, const float *scales, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, void *y,
                 int64_t y_stride, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    if (const int rc = check_product(c, "bs_w8_linear", weight, weight_scales, m, n, k, y, y_stride)) return rc;
    if (m == 0 || n == 0) return BS_OK;
    if (!q || !scales || !aligned16(q)) return ctx_fail(c, BS_EINVAL, "bs_w8_linear: rows are NULL or not 16-byte aligned");
    return products(c, (const int8_t *)q, scales, weight, weight_scales, m, n, k, y, y_stride, (hipStream_t)stream);
  });
}

int bs_w8_linear_rows(bs_ctx *c, const void *x, int64_t x_stride, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, void *y,
                      int64_t y_stride, void *scratch, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    if (const int rc = check_product(c, "bs_w8_linear_rows", weight, weight_scales, m, n, k, y, y_stride)) return rc;
    if (m == 0 || n == 0) return BS_OK;
    if (!x || x_stride < k || x_stride % 8 || !aligned16(x))
      return ctx_fail(c, BS_EINVAL, "bs_w8_linear_rows: rows of %lld elements at a stride of %lld (16-byte aligned, the stride a multiple of 8)", (long long)k, (long long)x_stride);
    if (few_rows(m, k)) {
      CTX_HIP_TRY(c, hipSetDevice(ctx_view(c).device));
      const int64_t most = MOST_BYTES / k / 256 * 256;
      for (int64_t n0 = 0; n0 < n; n0 += most) {
        const int64_t n1 = std::min(most, n - n0);
        FewArgs f{};
        f.g = product_args(c, nullptr, nullptr, (const int8_t *)weight + n0 * k, weight_scales + n0, (int)m, (int)n1, k, (uint16_t *)y + n0, y_stride);
        f.x = (const uint16_t *)x;
        f.x_stride = x_stride;
        CTX_HIP_TRY(c, launch_few_rows(f, few_blocks(n1, k, f.g.n_cu), (hipStream_t)stream));
      }
      return BS_OK;
    }
    const int64_t bytes = bs_w8_scratch_bytes(m, k);
    if ((bytes > 0 && !scratch) || !aligned16(scratch)) return ctx_fail(c, BS_EINVAL, "bs_w8_linear_rows: %lld bytes of scratch, 16-byte aligned", (long long)bytes);
    float *scales = (float *)scratch;
    int8_t *q = (int8_t *)scratch + (4 * m + 15) / 16 * 16;
    if (const int rc = bs_w8_quantize(c, x, x_stride, m, k, q, scales, stream)) return rc;
    return products(c, q, scales, weight, weight_scales, m, n, k, y, y_stride, (hipStream_t)stream);
  });
}

}  // extern "C"
