// Products of 8-bit integers with a scale for each row of either operand, and the rows' way there.
//
// y[m, n] = row_scale[m] col_scale[n] sum over k of xq[m, k] w[n, k]: sums of integers in 32 bits, exact whatever their order, then two products in
// 32 bits and one rounding.  v_mfma_i32_16x16x64_i8 takes the same 16 bytes of a row from a lane as the bf16 instruction of half the
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
  const bool bad = most >= 0x7F80u;  // a NaN or an infinity: the row's results are NaN
  const float scale = bad ? __builtin_nanf("") : fmaxf(__uint_as_float(most << 16), LEAST) / 127.f, inverse = 1.f / scale;
  if (threadIdx.x == 0) a.scale[row] = scale;
  int8_t *q = a.q + row * a.k;
  auto put = [&](u32x4_t v, int at) {
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
    *reinterpret_cast<u32x2_t *>(q + at) = u32x2_t{w[0], w[1]};
  };
#pragma unroll
  for (int i = 0; i < QUANT_KEPT; ++i) {
    const int at = (i * T + (int)threadIdx.x) * 8;
    if (at < a.k) put(kept[i], at);
  }
#pragma unroll 4
  for (int at = (QUANT_KEPT * T + (int)threadIdx.x) * 8; at < a.k; at += T * 8) put(attn_dev::ld16(x + at), at);
}

hipError_t launch_quantize(const QuantArgs &a, hipStream_t stream) {
  if (a.m <= 0) return hipSuccess;
  hipLaunchKernelGGL(w8_quantize_kernel<256>, dim3(a.m), dim3(256), 0, stream, a);
  return hipGetLastError();
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
  f32x4_t v = __builtin_convertvector(s, f32x4_t) * a.row_scale[m];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= a.col_scale[min(n + e, a.N - 1)];
  store_scaled4(a.C + (size_t)m * a.ldc + n, v, n, a.N, ((reinterpret_cast<uintptr_t>(a.C) | (uintptr_t)a.ldc * 2) & 7) == 0);
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

enum Shape { ROWS_11, ROWS_12, ROWS_21, ROWS_22, D64, D128, S128, S256, SMALL, WIDE, TALL, MID, BIG, N_SHAPES };
struct Plan {
  int shape, splits;
};

template <int EPI>
hipError_t launch_shape(int shape, const GemmArgs &a, hipStream_t stream) {
  switch (shape) {
    case D64: return launch_tiles<64, 128, 4, 2, EPI, 2>(a, stream);
    case D128: return launch_tiles<128, 128, 4, 2, EPI, 2>(a, stream);
    case S128: return launch_tiles<128, 256, 2, 4, EPI, 2>(a, stream);
    case S256: return launch_tiles<256, 128, 4, 2, EPI, 2>(a, stream);
    case SMALL: return launch_tiles<128, 128, 2, 2, EPI, 0>(a, stream);
    case WIDE: return launch_tiles<128, 256, 2, 4, EPI, 0>(a, stream);
    case TALL: return launch_tiles<160, 256, 2, 4, EPI, 0>(a, stream);
    case MID: return launch_tiles<192, 256, 2, 4, EPI, 0>(a, stream);
    case BIG: return launch_tiles<256, 256, 2, 4, EPI, 0>(a, stream);
  }
  return hipErrorInvalidValue;
}

Plan plan_of(int64_t m, int64_t n, int64_t k, int n_cu, size_t ws_floats) {
  if (m <= 16) return {ROWS_11, 1};
  if (m <= 32) return {ROWS_21, 1};
  if (m <= 64) return {D64, 1};
  if (m <= 128) return {D128, 1};
  return {BIG, 1};
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
constexpr int64_t MOST_K = 131072;          // 127 * 128 k stays in 32 bits
constexpr int64_t MOST_ROWS = 1 << 30;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

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

int bs_w8_linear(bs_ctx *c, const void *q, const float *scales, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, void *y,
                 int64_t y_stride, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    const CtxView v = ctx_view(c);
    if (v.device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
    if (m < 0 || m > MOST_ROWS || n < 0 || n > MOST_ROWS || k < 16 || k % 16 || k > MOST_K || y_stride > 0x7fffffff)
      return ctx_fail(c, BS_EUNSUPPORTED, "bs_w8_linear: m=%lld n=%lld k=%lld (k a multiple of 16 up to %lld), rows of y %lld apart", (long long)m, (long long)n,
                      (long long)k, (long long)MOST_K, (long long)y_stride);
    if (m == 0 || n == 0) return BS_OK;
    if (!q || !scales || !weight || !weight_scales || !y) return ctx_fail(c, BS_EINVAL, "bs_w8_linear: NULL pointer");
    if (y_stride < n || !aligned16(q) || !aligned16(weight))
      return ctx_fail(c, BS_EINVAL, "bs_w8_linear: rows of %lld elements at a stride of %lld (integers 16-byte aligned)", (long long)n, (long long)y_stride);
    CTX_HIP_TRY(c, hipSetDevice(v.device));
    // ranges of rows and of outputs whose operands offsets of 32 bits reach
    const int64_t most = MOST_BYTES / k / 256 * 256;
    for (int64_t m0 = 0; m0 < m; m0 += most)
      for (int64_t n0 = 0; n0 < n; n0 += most) {
        GemmArgs a{};
        a.A = (const uint16_t *)((const int8_t *)q + m0 * k);
        a.B = (const uint16_t *)((const int8_t *)weight + n0 * k);
        a.M = (int)std::min(most, m - m0);
        a.N = (int)std::min(most, n - n0);
        a.K = a.lda = a.ldb = (int)(k / 2);
        a.n_cu = v.n_cu;
        a.C = (uint16_t *)y + m0 * y_stride + n0;
        a.ldc = (int)y_stride;
        a.row_scale = scales + m0;
        a.col_scale = weight_scales + n0;
        a.sk_ws = v.ws;
        CTX_HIP_TRY(c, launch_product(a, v.ws_floats, (hipStream_t)stream));
      }
    return BS_OK;
  });
}

}  // extern "C"
