// Device code for workgroups that share a result: parts travel through memory, the last workgroup to arrive adds them up.
#pragma once
#include "common.hpp"

namespace bs {
namespace join_dev {

// 16-byte accesses that all XCDs agree on (their L2 caches are their own): parts travel past those.
constexpr int SC1 = 16;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t parts_of(const void *p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, 0x7fffffff, 0x00020000);
}
__device__ __forceinline__ void put_part(const __amdgpu_buffer_rsrc_t &rs, unsigned at, f32x4_t v) {
  const u32x4_t w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  __builtin_amdgcn_raw_buffer_store_b128(w, rs, at, 0, SC1);
}
__device__ __forceinline__ f32x4_t get_part(const __amdgpu_buffer_rsrc_t &rs, unsigned at) {
  const u32x4_t w = __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, SC1);
  return f32x4_t{__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
}

// Whether this workgroup is the last of `parts` to arrive at a counter, which it clears for the next launch.  Called by all of
// its threads; what they have put is where all XCDs see it before the workgroup counts itself in.
__device__ __forceinline__ bool last_of(unsigned *counter, unsigned parts, unsigned *flag) {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
  if (threadIdx.x == 0) *flag = atomicAdd(counter, 1u);
  __syncthreads();
  if (*flag + 1u != parts) return false;
  if (threadIdx.x == 0) atomicExch(counter, 0u);
  return true;
}

}  // namespace join_dev
}  // namespace bs
