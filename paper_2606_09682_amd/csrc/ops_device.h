// Device helpers shared by the operators for several tokens.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace amk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
// round to nearest, ties to even
__device__ __forceinline__ uint16_t f32_to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return (uint32_t)f32_to_bf16(lo) | (uint32_t)f32_to_bf16(hi) << 16;
}

#define AMK_LDS __attribute__((address_space(3)))

// 16 bytes a lane from global memory into 1 KiB of LDS at `lds` (the same for
// all lanes of the wave): lane i's bytes go to lds + 16 i.
__device__ __forceinline__ void load_lds16(const void* g, AMK_LDS void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g, lds, 16, 0, 0);
}

// Waits until at most N of this wave's loads, those to LDS among them, are under way
// (a barrier alone does not): they return in order.  The other counters stay at their maximum.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter has 6 bits");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

// The workgroup's barrier of a ring of stages: at most N loads of every wave are still
// under way behind it, and no read of LDS.  (A barrier with a fence would wait for all
// loads to LDS.)
template <int N>
__device__ __forceinline__ void stage_barrier() {
  static_assert(N < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Transposed LDS read: in each 16 lanes, lane i addresses 4 elements of row i / 4
// of a 4 x 16 block (columns 4 (i % 4) ..) and receives the block's column i.
__device__ __forceinline__ s16x4 read_tr16(const AMK_LDS uint16_t* lds) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((AMK_LDS s16x4*)lds);
}

// Reductions over a wave's 64 lanes in six steps within registers: shifts within rows of
// 16 lanes, then the rows' last lanes passed on.  Every lane gets the result.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float identity, float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, identity),
                                                               __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
template <typename Op>
__device__ __forceinline__ float wave_reduce(float v, float identity, Op op) {
  v = op(v, dpp<0x111, 0xf>(identity, v));
  v = op(v, dpp<0x112, 0xf>(identity, v));
  v = op(v, dpp<0x114, 0xf>(identity, v));
  v = op(v, dpp<0x118, 0xf>(identity, v));
  v = op(v, dpp<0x142, 0xa>(identity, v));
  v = op(v, dpp<0x143, 0xc>(identity, v));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.f, [](float a, float b) { return a + b; });
}

}  // namespace amk
