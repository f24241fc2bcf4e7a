// y = x W^T for several tokens, W in the decoder's weight formats.
//
// Both operands have their columns (k) contiguous, as the matrix instructions
// take them (32x32x16 bf16, sums in fp32).  x is the A operand and W the B operand: a
// lane's results lie in one row of W, so one scale serves all of them: W8A16
// multiplies the finished sums, W4A16 the sums over a group of columns.
//
// x and the raw bytes of W go straight to LDS (16 bytes a lane), two stages, a
// stage's loads under the other's products.  Codes become bf16 (exactly) in
// registers, after the read from LDS: a quantised W takes its smaller share of
// HBM, L2 and LDS alike, and the conversions of one wave run beside the products
// of another.  Rows lie without padding, their 16-byte chunks permuted by the row
// so that 16 rows read at one column meet in no bank.
//
// Columns within a slice of 32: a product's k slots 0..7 of lane half h in step s
// stand for columns 16 h + 8 s .. + 7, so that a lane's two steps are 32
// contiguous bytes of bf16, 16 of int8 or 8 of int4.
//
// Tiles.  A workgroup is WT x WR waves of (32 TB) tokens x (32 RB) rows of W, times KG
// groups of waves that share the tile and take a share of the columns each, joined
// through LDS at the end.  Long prompts need large tiles, few reads of LDS a product
// (KG 1); few tokens need the weights streamed by every CU, so small tiles and many
// waves on their columns.
#include "ops.h"
#include "ops_device.h"

namespace amk {
namespace {

__device__ __forceinline__ float half_to_f32(uint16_t h) { return (float)__builtin_bit_cast(_Float16, h); }

// bf16 of two floats that bf16 holds exactly
__device__ __forceinline__ uint32_t pack_exact(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}

// 8 int8 codes as bf16
__device__ __forceinline__ bf16x8 int8_to_bf16(uint32_t a, uint32_t b) {
  u32x4 r;
  r[0] = pack_exact((float)(int8_t)a, (float)(int8_t)(a >> 8));
  r[1] = pack_exact((float)(int8_t)(a >> 16), (float)(int8_t)(a >> 24));
  r[2] = pack_exact((float)(int8_t)b, (float)(int8_t)(b >> 8));
  r[3] = pack_exact((float)(int8_t)(b >> 16), (float)(int8_t)(b >> 24));
  return __builtin_bit_cast(bf16x8, r);
}

// The 8 codes of one packed int4 word: low nibbles are columns 0..3, high ones 4..7.
__device__ __forceinline__ bf16x8 int4_to_bf16(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  u32x4 r;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t n = (p < 2 ? lo : hi) >> (p % 2 * 16);
    r[p] = pack_exact((float)(n & 0xffu) - 8.f, (float)((n >> 8) & 0xffu) - 8.f);
  }
  return __builtin_bit_cast(bf16x8, r);
}

template <int FMT, int TB_, int RB_, int WT_, int WR_, int KG_, int BKW_>
struct Tile {
  static constexpr int TB = TB_, RB = RB_, WT = WT_, WR = WR_, KG = KG_, BKW = BKW_;
  static constexpr int WAVES = WT * WR * KG, THREADS = 64 * WAVES;
  static constexpr int BT = 32 * TB * WT, BR = 32 * RB * WR;  // tokens, rows of W
  static constexpr int COLS = KG * BKW;                       // columns of a stage
  static constexpr int EIGHT = FMT == AMK_WEIGHTS_BF16 ? 16 : FMT == AMK_WEIGHTS_W8A16 ? 8 : 4;  // bytes of 8 columns of W
  static constexpr int XC = BKW / 8, WC = BKW * EIGHT / 128;  // 16-byte chunks per row of a slice
  static constexpr int XCHUNKS = KG * BT * XC, WCHUNKS = KG * BR * WC;
  static constexpr int XLOADS = XCHUNKS / THREADS, WLOADS = WCHUNKS / THREADS;
  static constexpr int STAGE = 16 * (XCHUNKS + WCHUNKS);
  static constexpr int JOIN = KG > 1 ? KG * TB * RB * 4096 : 0;  // sums of all column groups
  static constexpr int LDS = 2 * STAGE > JOIN ? 2 * STAGE : JOIN;
  static_assert(XCHUNKS % THREADS == 0 && WCHUNKS % THREADS == 0 && WLOADS > 0 && XLOADS > 0, "whole loads");
  static_assert(KG == 1 || (WT == 1 && WR == 1), "column groups share one tile");
};

// Permutation of the C chunks of a row: rows that share a bank row of 256 bytes differ.
template <int C>
__device__ __forceinline__ int swizzle(int row) {
  return row / (16 / C) % C;
}

// Loads one stage: columns k0 .. of the tile's rows.  Rows past the last repeat it and
// columns past the last the first ones: in range, and their results are not used.
template <int FMT, typename G>
__device__ __forceinline__ void load_stage(const LinearArgs& a, int t0, int r0, int k0,
                                           AMK_LDS unsigned char* to) {
  AMK_LDS unsigned char* dst = to + threadIdx.x / 64 * 1024;
#pragma unroll
  for (int i = 0; i < G::XLOADS; ++i) {
    const int c = i * G::THREADS + threadIdx.x, at = c % G::XC, row = c / G::XC % G::BT, kg = c / (G::XC * G::BT);
    int k = k0 + kg * G::BKW + (at ^ swizzle<G::XC>(row)) * 8;
    k = k < a.in ? k : 0;
    load_lds16(a.x + (int64_t)min(t0 + row, a.n - 1) * a.x_stride + k, dst + i * G::THREADS * 16);
  }
#pragma unroll
  for (int i = 0; i < G::WLOADS; ++i) {
    const int c = i * G::THREADS + threadIdx.x, at = c % G::WC, row = c / G::WC % G::BR, kg = c / (G::WC * G::BR);
    int k = k0 + kg * G::BKW + (at ^ swizzle<G::WC>(row)) * (128 / G::EIGHT);
    k = k < a.in ? k : 0;
    const int64_t eight = ((int64_t)min(r0 + row, a.out - 1) * a.in + k) / 8;
    load_lds16((const unsigned char*)a.w + eight * G::EIGHT, dst + (G::XCHUNKS + i * G::THREADS) * 16);
  }
}

// The products of this wave's share of one stage.  xs, ws and next do not overlap: without
// that promise every read would wait for the loads of the next stage.
template <int FMT, typename G, bool TAIL, bool GROUP32>
__device__ __forceinline__ void linear_step(const LinearArgs& a, int t0, int r0, int k0, bool more,
                                            const AMK_LDS unsigned char* __restrict__ xs,
                                            const AMK_LDS unsigned char* __restrict__ ws,
                                            AMK_LDS unsigned char* __restrict__ next, const float (&scale)[G::RB][2],
                                            f32x16 (&acc)[G::TB][G::RB], f32x16 (&part)[G::TB][G::RB]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
  const int kg = wave / (G::WT * G::WR), wt = wave % G::WT, wr = wave / G::WT % G::WR;
  const int kw = k0 + kg * G::BKW;  // the wave's first column
  if (more) load_stage<FMT, G>(a, t0, r0, k0 + G::COLS, next);
  xs += (kg * G::BT + wt * 32 * G::TB + col) * G::XC * 16;
  ws += (kg * G::BR + wr * 32 * G::RB + col) * G::WC * 16;
#pragma unroll
  for (int u = 0; u < G::BKW / 32; ++u) {
    bf16x8 xf[G::TB][2], wf[G::RB][2];
#pragma unroll
    for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int row = 32 * tb + col, c = (4 * u + 2 * half + s) ^ swizzle<G::XC>(row);
        xf[tb][s] = *(const AMK_LDS bf16x8*)(xs + 32 * tb * G::XC * 16 + c * 16);
        if (TAIL && kw + 32 * u + 16 * half + 8 * s >= a.in) xf[tb][s] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
      }
#pragma unroll
    for (int rb = 0; rb < G::RB; ++rb) {
      const AMK_LDS unsigned char* wrow = ws + 32 * rb * G::WC * 16;
      const int sw = swizzle<G::WC>(32 * rb + col);
      if constexpr (FMT == AMK_WEIGHTS_BF16) {
#pragma unroll
        for (int s = 0; s < 2; ++s) wf[rb][s] = *(const AMK_LDS bf16x8*)(wrow + ((4 * u + 2 * half + s) ^ sw) * 16);
      } else if constexpr (FMT == AMK_WEIGHTS_W8A16) {
        const u32x4 v = *(const AMK_LDS u32x4*)(wrow + ((2 * u + half) ^ sw) * 16);
        wf[rb][0] = int8_to_bf16(v[0], v[1]);
        wf[rb][1] = int8_to_bf16(v[2], v[3]);
      } else {
        const u32x2 v = *(const AMK_LDS u32x2*)(wrow + (u ^ sw) * 16 + half * 8);
        wf[rb][0] = int4_to_bf16(v[0]);
        wf[rb][1] = int4_to_bf16(v[1]);
      }
    }
    if constexpr (TAIL) {  // W's too: 0 times what lies there need not be 0
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (kw + 32 * u + 16 * half + 8 * s >= a.in) wf[rb][s] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    }
    f32x16(&sum)[G::TB][G::RB] = FMT == AMK_WEIGHTS_W4A16 ? part : acc;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
        for (int rb = 0; rb < G::RB; ++rb)
          sum[tb][rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[tb][s], wf[rb][s], sum[tb][rb], 0, 0, 0);
    if constexpr (FMT == AMK_WEIGHTS_W4A16) {
      // a group of columns is complete: at the end of the slice, where the next one is
      // another's (column groups of waves), or at the group's end
      const bool last = u + 1 == G::BKW / 32;
      if (GROUP32 || (last && (G::KG > 1 || ((kw + G::BKW) & (a.group - 1)) == 0 || TAIL))) {
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
          for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              acc[tb][rb][i] = __builtin_fmaf(scale[rb][GROUP32 ? u : 0], part[tb][rb][i], acc[tb][rb][i]);
              part[tb][rb][i] = 0.f;
            }
      }
    }
  }
}

__device__ __forceinline__ void put(const LinearArgs& a, int t, int r, float y) {
  const int64_t at = t * a.y_stride + r;
  if (a.y_bf16) {
    uint16_t* p = (uint16_t*)a.y + at;
    *p = f32_to_bf16(a.accumulate ? bf16_to_f32(*p) + y : y);
  } else {
    float* p = (float*)a.y + at;
    *p = a.accumulate ? *p + y : y;
  }
}

template <int FMT, typename G, bool GROUP32>
__global__ void __launch_bounds__(G::THREADS, 2) linear_kernel(const LinearArgs a, int token_tiles, int row_tiles) {
  __shared__ __align__(16) unsigned char lds[G::LDS];
  AMK_LDS unsigned char* mem = (AMK_LDS unsigned char*)lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
  const int kg = wave / (G::WT * G::WR), wt = wave % G::WT, wr = wave / G::WT % G::WR;
  // Workgroups go to the 8 XCDs in turn: each XCD takes a run of tiles, token tiles of
  // one stretch of W first, so that its L2 reads those rows once.
  const int tiles = token_tiles * row_tiles, each = (tiles + 7) / 8;
  const int tile = (int)(blockIdx.x % 8) * each + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= each || tile >= tiles) return;
  const int t0 = tile % token_tiles * G::BT, r0 = tile / token_tiles * G::BR;

  // this lane's rows of W and, under W4A16, their scales of the next stage's groups
  const uint16_t* srow[G::RB];
  const int groups = FMT == AMK_WEIGHTS_W4A16 ? a.in / a.group : 0;
#pragma unroll
  for (int rb = 0; rb < G::RB; ++rb)
    srow[rb] = (const uint16_t*)a.scale + (int64_t)min(r0 + (wr * G::RB + rb) * 32 + col, a.out - 1) * groups;
  const int shift = FMT == AMK_WEIGHTS_W4A16 ? __builtin_ctz(a.group) : 0;
  uint16_t ahead[G::RB][2] = {};
  auto fetch = [&](int k0) {
    if constexpr (FMT == AMK_WEIGHTS_W4A16) {
      const int kw = k0 + kg * G::BKW;
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int u = 0; u < (GROUP32 ? G::BKW / 32 : 1); ++u)
          ahead[rb][u] = srow[rb][min((kw + 32 * u) >> shift, groups - 1)];
    }
  };

  f32x16 acc[G::TB][G::RB] = {}, part[G::TB][G::RB] = {};
  fetch(0);
  load_stage<FMT, G>(a, t0, r0, 0, mem);
  int stage = 0, k0 = 0;
  for (; k0 + G::COLS <= a.in; k0 += G::COLS, stage ^= 1) {
    wait_loads();
    __syncthreads();  // the stage is in, and the readers of the other one are done
    float scale[G::RB][2] = {};
    if constexpr (FMT == AMK_WEIGHTS_W4A16) {
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int u = 0; u < 2; ++u) scale[rb][u] = half_to_f32(ahead[rb][u]);
      fetch(k0 + G::COLS);
    }
    AMK_LDS unsigned char* cur = mem + stage * G::STAGE;
    linear_step<FMT, G, false, GROUP32>(a, t0, r0, k0, k0 + G::COLS < a.in, cur, cur + 16 * G::XCHUNKS,
                                        mem + (stage ^ 1) * G::STAGE, scale, acc, part);
  }
  if (k0 < a.in) {
    wait_loads();
    __syncthreads();
    float scale[G::RB][2] = {};
    if constexpr (FMT == AMK_WEIGHTS_W4A16) {
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int u = 0; u < 2; ++u) scale[rb][u] = half_to_f32(ahead[rb][u]);
    }
    AMK_LDS unsigned char* cur = mem + stage * G::STAGE;
    linear_step<FMT, G, true, GROUP32>(a, t0, r0, k0, false, cur, cur + 16 * G::XCHUNKS, mem + (stage ^ 1) * G::STAGE,
                                       scale, acc, part);
  }

  if constexpr (G::KG == 1) {
#pragma unroll
    for (int rb = 0; rb < G::RB; ++rb) {
      const int r = r0 + (wr * G::RB + rb) * 32 + col;
      if (r >= a.out) continue;
      const float sc = FMT == AMK_WEIGHTS_W8A16 ? ((const float*)a.scale)[r] : 1.f;
#pragma unroll
      for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = t0 + (wt * G::TB + tb) * 32 + 8 * (i / 4) + 4 * half + i % 4;
          if (t < a.n) put(a, t, r, acc[tb][rb][i] * sc);
        }
    }
  } else {
    // add up the column groups in order
    constexpr int BLOCKS = G::TB * G::RB;
    AMK_LDS float* sums = (AMK_LDS float*)mem;
    __syncthreads();
#pragma unroll
    for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sums[((kg * BLOCKS + tb * G::RB + rb) * 16 + i) * 64 + lane] = acc[tb][rb][i];
    __syncthreads();
    for (int o = threadIdx.x; o < BLOCKS * 1024; o += G::THREADS) {
      const int l = o % 64, i = o / 64 % 16, rb = o / 1024 % G::RB, tb = o / 1024 / G::RB;
      const int t = t0 + tb * 32 + 8 * (i / 4) + 4 * (l / 32) + i % 4, r = r0 + rb * 32 + l % 32;
      if (t >= a.n || r >= a.out) continue;
      float y = sums[o];
      for (int g = 1; g < G::KG; ++g) y += sums[g * BLOCKS * 1024 + o];
      put(a, t, r, FMT == AMK_WEIGHTS_W8A16 ? y * ((const float*)a.scale)[r] : y);
    }
  }
}

template <int FMT, typename G>
int launch_tile(const LinearArgs& a, hipStream_t st) {
  const int tt = (a.n + G::BT - 1) / G::BT, rt = (a.out + G::BR - 1) / G::BR;
  const dim3 grid((unsigned)(((int64_t)tt * rt + 7) / 8 * 8));
  if (FMT == AMK_WEIGHTS_W4A16 && a.group == 32)
    hipLaunchKernelGGL((linear_kernel<FMT, G, FMT == AMK_WEIGHTS_W4A16>), grid, dim3(G::THREADS), 0, st, a, tt, rt);
  else
    hipLaunchKernelGGL((linear_kernel<FMT, G, false>), grid, dim3(G::THREADS), 0, st, a, tt, rt);
  return hipGetLastError() == hipSuccess ? AMK_OK : AMK_ERR_DEVICE;
}

template <int FMT>
int launch_fmt(const LinearArgs& a, hipStream_t st) {
  constexpr bool W4 = FMT == AMK_WEIGHTS_W4A16;
  const int64_t large = (int64_t)((a.n + 255) / 256) * ((a.out + 255) / 256);
  if (a.n <= 32) return launch_tile<FMT, Tile<FMT, 1, 1, 1, 1, 8, W4 ? 64 : 32>>(a, st);
  if (large < 128) return launch_tile<FMT, Tile<FMT, 2, 2, 1, 1, 8, W4 ? 64 : 32>>(a, st);
  return launch_tile<FMT, Tile<FMT, W4 ? 2 : 4, 2, 2, 4, 1, 64>>(a, st);
}

}  // namespace

int launch_linear(const LinearArgs& a, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (a.fmt == AMK_WEIGHTS_BF16) return launch_fmt<AMK_WEIGHTS_BF16>(a, st);
  if (a.fmt == AMK_WEIGHTS_W8A16) return launch_fmt<AMK_WEIGHTS_W8A16>(a, st);
  return launch_fmt<AMK_WEIGHTS_W4A16>(a, st);
}

}  // namespace amk
