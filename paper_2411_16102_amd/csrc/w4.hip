// Products of few rows with 4-bit weights that have a scale per group of inputs.
//
//   y[m, n] = sum_g scale[n, g] * (sum_{k in g} x[m, k] w[n, k] - zero[n, g] sum_{k in g} x[m, k])
//
// The weights become bf16 matrix operands without arithmetic: 0x4300 | w is the bf16 number 128 + w (its last mantissa
// bit counts 1), so a shift and an and-or make two of them, and
//   sum x w = sum x (128 + w) - 128 sum x,
// which joins the zero point: y += scale * (D - (128 + zero) * X), D the product over the group and X the sum of its x.  All in 32 bits:
// D is at most some hundred times the result, which leaves 16 of its 24 bits.
#include "../../include/blendstep_stream.h"
#include "common.hpp"
#include "context.hpp"
#include "w4.hpp"

using namespace bs;

namespace bs {
namespace {

__device__ __forceinline__ bf16x8_t as_operand(uint32_t w) {
  constexpr uint32_t MASK = 0x000F000Fu, BASE = 0x43004300u;
  const u32x4_t v = {(w & MASK) | BASE, ((w >> 4) & MASK) | BASE, ((w >> 8) & MASK) | BASE, ((w >> 12) & MASK) | BASE};
  return as_bf16x8(v);
}

// A wavefront per 16 outputs and 16 rows.
template <int GROUP, bool ZEROS>
__global__ __launch_bounds__(64) void w4_kernel(const W4Args a, const W4Layout l) {
  constexpr int STEPS = GROUP / 32;  // matrix instructions of a group
  const int lane = threadIdx.x & 63, j = lane & 15, g4 = lane >> 4;
  const int64_t nb = blockIdx.x;
  const int m = blockIdx.y * 16 + j;
  const uint16_t *x = a.x + m * a.x_stride + 8 * g4;
  const u32x4_t ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  f32x4_t y = {0.f, 0.f, 0.f, 0.f};
  for (int64_t kb = 0; kb < l.k_blocks; ++kb) {
    const u32x4_t w = *reinterpret_cast<const u32x4_t *>(a.weight + (nb * l.k_blocks + kb) * 1024 + lane * 16);
#pragma unroll
    for (int g = 0; g < 128 / GROUP; ++g) {
      const int64_t at = nb * l.groups + kb * (128 / GROUP) + g;
      f32x4_t d = {0.f, 0.f, 0.f, 0.f}, sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int k0 = (int)kb * 128 + (g * STEPS + s) * 32;
        u32x4_t xv = {0u, 0u, 0u, 0u};
        if (m < a.m && k0 < a.k) xv = *reinterpret_cast<const u32x4_t *>(x + k0);  // (k is a multiple of 32)
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_operand(w[g * STEPS + s]), as_bf16x8(xv), d, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(ones), as_bf16x8(xv), sum, 0, 0, 0);
      }
      const u32x2_t sc = *reinterpret_cast<const u32x2_t *>(a.weight + l.scales + at * 32 + 8 * g4);
      const uint32_t z = ZEROS ? *reinterpret_cast<const uint32_t *>(a.weight + l.zeros + at * 16 + 4 * g4) : 0x08080808u;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float s = __uint_as_float(r & 1 ? sc[r >> 1] & 0xFFFF0000u : sc[r >> 1] << 16);
        y[r] += s * (d[r] - (128.f + (float)((z >> (8 * r)) & 0xFFu)) * sum[r]);
      }
    }
  }
  if (m >= a.m) return;
  const int64_t n0 = nb * 16 + 4 * g4;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n0 + r < a.n) a.y[m * a.y_stride + n0 + r] = (uint16_t)pack_bf16x2(y[r], 0.f);
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
  const int64_t row = e / 16 / l.groups * 16 + e % 16, g = e / 16 % l.groups;
  const bool in = row < n && g * group < k;
  reinterpret_cast<uint16_t *>(weight + l.scales)[e] = in ? scales[row * (k / group) + g] : (uint16_t)0;
  if (zeros) weight[l.zeros + e] = in ? zeros[row * (k / group) + g] : (unsigned char)0;
}

template <int GROUP>
hipError_t launch_group(const W4Args &a, const W4Layout &l, hipStream_t stream) {
  const dim3 grid((unsigned)l.n_blocks, (unsigned)((a.m + 15) / 16));
  if (a.with_zeros) hipLaunchKernelGGL((w4_kernel<GROUP, true>), grid, dim3(64), 0, stream, a, l);
  else hipLaunchKernelGGL((w4_kernel<GROUP, false>), grid, dim3(64), 0, stream, a, l);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w4_linear(const W4Args &a, hipStream_t stream) {
  if (a.m <= 0 || a.n <= 0) return hipSuccess;
  const W4Layout l = w4_layout(a.n, a.k, a.group, a.with_zeros);
  if (a.group == 32) return launch_group<32>(a, l, stream);
  if (a.group == 64) return launch_group<64>(a, l, stream);
  if (a.group == 128) return launch_group<128>(a, l, stream);
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
    if (!shape_ok(n, k, group) || m < 0 || m > 65535 * 16)
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
    CTX_HIP_TRY(c, launch_w4_linear(a, (hipStream_t)stream));
    return BS_OK;
  });
}

}  // extern "C"
