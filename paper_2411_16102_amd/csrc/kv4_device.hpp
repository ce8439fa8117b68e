// Codes of a cache in four bits (see kv4.hpp): making them and reading them.
#pragma once
#include "common.hpp"
#include "kv4.hpp"

namespace bs {
namespace kv4_dev {

constexpr float CENTRE = 24.f;  // 16 + code less this is code - 8

__device__ __forceinline__ uint32_t turn_left3(uint32_t w) { return __builtin_amdgcn_alignbit(w, w, 29); }

// The eight elements of a word as bf16 numbers 16 + code.  Bits 3 to 6 of a bf16 number between 16 and 32 count whole numbers.  The two constants are
// in registers of their own, so that an and and an or are one instruction (which takes one constant at most).
struct Unpack {
  uint32_t codes, sixteens;
  __device__ __forceinline__ Unpack() {
    asm("s_mov_b32 %0, 0x780078" : "=s"(codes));
    asm("v_mov_b32 %0, 0x41804180" : "=v"(sixteens));
  }
  __device__ __forceinline__ u32x4_t operator()(uint32_t w) const {
    return u32x4_t{(w & codes) | sixteens, ((w >> 4) & codes) | sixteens, ((w >> 8) & codes) | sixteens, (__builtin_amdgcn_alignbit(w, w, 12) & codes) | sixteens};
  }
};

// element j of a word
__device__ __forceinline__ uint32_t code_of(uint32_t w, int j) { return (__builtin_amdgcn_alignbit(w, w, 3) >> (4 * (j >> 1) + 16 * (j & 1))) & 15u; }

// eight codes as a word
__device__ __forceinline__ uint32_t word_of(const uint32_t (&c)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) w |= c[j] << (4 * (j >> 1) + 16 * (j & 1));
  return turn_left3(w);
}

// what code c stands for, in 32 bits (the product is exact: 8 bits by 4)
__device__ __forceinline__ float value_of(float scale, float mid, uint32_t c) { return __builtin_fmaf(scale, (float)((int)c - 8), mid); }

// The numbers of a group: mid is the place of code 8 where 0 .. 15 span [lo, hi], rounded to bf16; scale the smallest bf16 number with which the
// codes still reach lo and hi, so that no value is further than half a scale from what its code stands for.  A group
// that holds a NaN or an infinity, or spans more than 32 bits can say, stands for NaN throughout.
struct Numbers {
  float scale, mid, inverse;  // inverse: 1 / scale, correctly rounded
  bool bad;
};
__device__ __forceinline__ Numbers numbers_of(float lo, float hi, bool bad) {
#pragma clang fp contract(off)
  Numbers n;
  n.mid = round_bf16(lo + 8.f * ((hi - lo) / 15.f));
  const float want = fmaxf((n.mid - lo) * 0.125f, (hi - n.mid) / 7.f);
  n.scale = fmaxf(__uint_as_float((__float_as_uint(want) + 0xFFFFu) & 0xFFFF0000u), 1.17549435e-38f);  // (2^-126: codes of equal values are finite)
  n.bad = bad | !(hi - lo < __builtin_inff()) | !(fabsf(n.mid) < __builtin_inff());
  n.inverse = 1.f / n.scale;
  return n;
}
__device__ __forceinline__ uint32_t scale_bits(const Numbers &n) { return n.bad ? 0x7FC0u : __float_as_uint(n.scale) >> 16; }
__device__ __forceinline__ uint32_t mid_bits(const Numbers &n) { return n.bad ? 0u : __float_as_uint(n.mid) >> 16; }

// The nearest code, ties to even.  The quotient is rounded correctly (its residual is exact), since values that came from bf16 often
// lie halfway between two codes.
__device__ __forceinline__ uint32_t code_for(const Numbers &n, float v) {
#pragma clang fp contract(off)
  const float a = v - n.mid;
  float q = a * n.inverse;
  q = __builtin_fmaf(__builtin_fmaf(-q, n.scale, a), n.inverse, q);
  const float c = __builtin_amdgcn_fmed3f(__builtin_rintf(q) + 8.f, 0.f, 15.f);
  return n.bad ? 0u : (uint32_t)c;
}

}  // namespace kv4_dev
}  // namespace bs
