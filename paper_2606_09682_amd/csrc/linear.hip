// y = x W^T for several tokens, W in the decoder's weight formats.
//
// A workgroup takes 64 tokens x 64 rows of W, a wave 32 x 32 of them, in steps of
// 64 columns.  x (bf16) and W's codes (bf16 weights as they are, int8 and int4
// codes converted, which bf16 holds exactly) are staged in LDS; the products are
// 32x32x16 matrix instructions summed in fp32.  Rows of W are the columns of a
// wave's tile, so a lane holds one row of W: its scale multiplies the finished
// sum (W8A16), or the sum of each 32 columns, whose group has one scale (W4A16).
#include "ops.h"
#include "ops_device.h"

namespace amk {
namespace {

constexpr int BT = 64, BR = 64, BK = 64;  // tokens, rows of W, columns of one step
constexpr int PITCH = BK + 8;             // LDS row pitch in elements

__device__ __forceinline__ float half_to_f32(uint16_t h) { return (float)__builtin_bit_cast(_Float16, h); }

// The 8 codes of one packed int4 word as bf16: low nibbles are columns 0..3, high ones 4..7.
__device__ __forceinline__ u32x4 int4_to_bf16(uint32_t w) {
  u32x4 r;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t n = p < 2 ? w : w >> 4;
    const int at = (p & 1) * 16;
    r[p] = pack_bf16((float)((int)(n >> at & 15) - 8), (float)((int)(n >> (at + 8) & 15) - 8));
  }
  return r;
}

__device__ __forceinline__ u32x4 int8_to_bf16(u32x2 w) {
  u32x4 r;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t v = w[p / 2];
    const int at = (p & 1) * 16;
    r[p] = pack_bf16((float)(int8_t)(v >> at), (float)(int8_t)(v >> (at + 8)));
  }
  return r;
}

// 8 columns of a row of W from column c (a multiple of 8) as bf16
template <int FMT>
__device__ __forceinline__ u32x4 load_w(const void* w, int64_t row, int in, int c) {
  if (FMT == AMK_WEIGHTS_BF16) return *(const u32x4*)((const uint16_t*)w + row * in + c);
  if (FMT == AMK_WEIGHTS_W8A16) return int8_to_bf16(*(const u32x2*)((const uint8_t*)w + row * in + c));
  return int4_to_bf16(*(const uint32_t*)((const uint8_t*)w + (row * in + c) / 2));
}

template <int FMT>
__global__ void __launch_bounds__(256) linear_tile_kernel(const LinearArgs a) {
  __shared__ __align__(16) uint16_t xs[BT * PITCH], ws[BR * PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int half = lane >> 5, col = lane & 31;
  const int r0 = blockIdx.x * BR, t0 = blockIdx.y * BT;
  const int wt = (wave & 1) * 32, wr = (wave >> 1) * 32;
  const int row = r0 + wr + col;
  const int srow = min(row, a.out - 1);
  f32x16 acc = {};
  for (int k0 = 0; k0 < a.in; k0 += BK) {
    __syncthreads();
    for (int c = threadIdx.x; c < BT * BK / 8; c += 256) {
      const int r = c / (BK / 8), k = k0 + c % (BK / 8) * 8;
      u32x4 x = {0, 0, 0, 0}, w = {0, 0, 0, 0};
      if (k < a.in) {
        x = *(const u32x4*)(a.x + (int64_t)min(t0 + r, a.n - 1) * a.x_stride + k);
        w = load_w<FMT>(a.w, min(r0 + r, a.out - 1), a.in, k);
      }
      *(u32x4*)(xs + r * PITCH + c % (BK / 8) * 8) = x;
      *(u32x4*)(ws + r * PITCH + c % (BK / 8) * 8) = w;
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < BK / 32; ++g) {
      f32x16 part = {};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = g * 32 + i * 16 + half * 8;
        const bf16x8 xf = *(const bf16x8*)(xs + (wt + col) * PITCH + k);
        const bf16x8 wf = *(const bf16x8*)(ws + (wr + col) * PITCH + k);
        if (FMT == AMK_WEIGHTS_W4A16) part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf, wf, part, 0, 0, 0);
        else acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf, wf, acc, 0, 0, 0);
      }
      if (FMT == AMK_WEIGHTS_W4A16 && k0 + g * 32 < a.in) {
        const float sc = half_to_f32(((const uint16_t*)a.scale)[(int64_t)srow * (a.in / a.group) + (k0 + g * 32) / a.group]);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] += sc * part[i];
      }
    }
  }
  if (row >= a.out) return;
  const float sc = FMT == AMK_WEIGHTS_W8A16 ? ((const float*)a.scale)[row] : 1.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int t = t0 + wt + 8 * (i / 4) + 4 * half + i % 4;
    if (t >= a.n) continue;
    float y = acc[i] * sc;
    const int64_t at = t * a.y_stride + row;
    if (a.y_bf16) {
      uint16_t* p = (uint16_t*)a.y + at;
      *p = f32_to_bf16(a.accumulate ? bf16_to_f32(*p) + y : y);
    } else {
      float* p = (float*)a.y + at;
      *p = a.accumulate ? *p + y : y;
    }
  }
}

}  // namespace

int launch_linear(const LinearArgs& a, void* stream) {
  const dim3 grid((a.out + BR - 1) / BR, (a.n + BT - 1) / BT);
  hipStream_t st = (hipStream_t)stream;
  if (a.fmt == AMK_WEIGHTS_BF16) hipLaunchKernelGGL(linear_tile_kernel<AMK_WEIGHTS_BF16>, grid, dim3(256), 0, st, a);
  else if (a.fmt == AMK_WEIGHTS_W8A16) hipLaunchKernelGGL(linear_tile_kernel<AMK_WEIGHTS_W8A16>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(linear_tile_kernel<AMK_WEIGHTS_W4A16>, grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? AMK_OK : AMK_ERR_DEVICE;
}

}  // namespace amk
