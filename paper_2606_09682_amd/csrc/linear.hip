// y = x W^T for several tokens, W in the decoder's weight formats.
//
// Both operands have their columns (k) contiguous, as the matrix instructions
// take them (32x32x16 bf16, sums in fp32).  x is the A operand and W the B operand: a
// lane's results lie in one row of W, so one scale serves all of them: W8A16
// multiplies the finished sums, W4A16 the sums over a group of columns.
//
// x and the raw bytes of W go straight to LDS (16 bytes a lane), two or three stages,
// the loads of one or two under the products of another.  Codes become bf16 (exactly) in
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
// waves on their columns.  A launch may take up to three matrices that x is multiplied
// with (Q, K and V; gate and up), whose tiles fill the CUs together.
//
// What bounds it.  2048 tokens 4096 -> 14336: matrix cores (busy 55% of the time; 448
// tiles of 256 x 256 are 1.75 rounds of the CUs), bf16 232 us, 1035 TFLOP/s (the library's
// product 208, a large square one 1380); int8 240; int4, which also converts and scales
// sums, 300.  32 tokens 4096 -> 14336: bf16 27 us (4.4 TB/s), int8 13.7, int4 13.9: with
// the smaller formats the copies of x that every tile reads from L2, 117 MB, weigh more
// than the weights.  5 tokens int8 576 -> 1536 take 3.6 us, hardly more than a launch.
#include <type_traits>

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

// The 8 codes of one packed int4 word as bf16 (low nibbles are columns 0..3, high ones 4..7;
// a nibble u stands for c = u - 8).  A byte of a sign and |c| <= 8, read as FP8 E4M3, is c
// steps of its subnormals (8 is the first normal number), 2^-9 each, which the conversion's
// scale makes 1: less work than a conversion through fp32.
__device__ __forceinline__ bf16x8 int4_to_bf16(uint32_t w) {
  const uint32_t sign = ~w & 0x88888888u;            // of each nibble
  const uint32_t neg = sign >> 3;
  const uint32_t mag = (w ^ (0x88888888u - neg)) + neg;  // u - 8, or (u ^ 7) + 1 = 8 - u: within the nibble
  const uint32_t lo = (mag & 0x0f0f0f0fu) | ((sign << 4) & 0xf0f0f0f0u);
  const uint32_t hi = ((mag >> 4) & 0x0f0f0f0fu) | (sign & 0xf0f0f0f0u);
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 r;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true);
  r[0] = __builtin_bit_cast(uint32_t, a);
  r[1] = __builtin_bit_cast(uint32_t, b);
  r[2] = __builtin_bit_cast(uint32_t, c);
  r[3] = __builtin_bit_cast(uint32_t, d);
  return __builtin_bit_cast(bf16x8, r);
}

template <int FMT, int TB_, int RB_, int WT_, int WR_, int KG_, int BKW_, int STAGES_ = 2, int XR_ = 32 * TB_ * WT_>
struct Tile {
  static constexpr int TB = TB_, RB = RB_, WT = WT_, WR = WR_, KG = KG_, BKW = BKW_;
  static constexpr int STAGES = STAGES_, XR = XR_;            // ring of stages, rows of x in each
  static constexpr int WAVES = WT * WR * KG, THREADS = 64 * WAVES;
  static constexpr int BT = 32 * TB * WT, BR = 32 * RB * WR;  // tokens, rows of W
  static constexpr int COLS = KG * BKW;                       // columns of a stage
  static constexpr int EIGHT = FMT == AMK_WEIGHTS_BF16 ? 16 : FMT == AMK_WEIGHTS_W8A16 ? 8 : 4;  // bytes of 8 columns of W
  static constexpr int XC = BKW / 8, WC = BKW * EIGHT / 128;  // 16-byte chunks per row of a slice
  static constexpr int XCHUNKS = KG * XR * XC, WCHUNKS = KG * BR * WC;
  static constexpr int XLOADS = XCHUNKS / THREADS, WLOADS = WCHUNKS / THREADS;
  static constexpr int STAGE = 16 * (XCHUNKS + WCHUNKS);
  static constexpr int JOIN = KG > 1 ? KG * TB * RB * 4096 : 0;  // sums of all column groups
  static constexpr int LDS = STAGES * STAGE > JOIN ? STAGES * STAGE : JOIN;
  static_assert(XCHUNKS % THREADS == 0 && WCHUNKS % THREADS == 0 && WLOADS > 0 && XLOADS > 0, "whole loads");
  static_assert(KG == 1 || (WT == 1 && WR == 1), "column groups share one tile");
  static_assert(XR == BT || TB * WT == 1, "rows of x repeat in the only block of tokens");
};

// Permutation of the C chunks of a row: rows that share a bank row of 256 bytes differ.
template <int C>
__device__ __forceinline__ int swizzle(int row) {
  return row / (16 / C) % C;
}

// This lane's loads of a stage: its 16 bytes of each lie in row `row` of the tile, at
// column `k` of the stage.
template <typename G>
struct Lane {
  int row, k;
  static __device__ __forceinline__ Lane x(int i) {
    const int c = i * G::THREADS + threadIdx.x, row = c / G::XC % G::XR;
    return {row, c / (G::XC * G::XR) * G::BKW + (c % G::XC ^ swizzle<G::XC>(row)) * 8};
  }
  static __device__ __forceinline__ Lane w(int i) {
    const int c = i * G::THREADS + threadIdx.x, row = c / G::WC % G::BR;
    return {row, c / (G::WC * G::BR) * G::BKW + (c % G::WC ^ swizzle<G::WC>(row)) * (128 / G::EIGHT)};
  }
};

// The tile's first rows of x and W, and the bytes from there to the rows of this lane's
// loads (rows past the last repeat it) at column 0 of a stage.
template <typename G>
struct Source {
  const unsigned char *x, *w;
  uint32_t xo[G::XLOADS], wo[G::WLOADS];

  __device__ __forceinline__ Source(const LinearArgs& a, const LinearPart& p, int t0, int r0) {
    x = (const unsigned char*)(a.x + (int64_t)t0 * a.x_stride);
    w = (const unsigned char*)p.w + (int64_t)r0 * (a.in / 8) * G::EIGHT;
#pragma unroll
    for (int i = 0; i < G::XLOADS; ++i) {
      const Lane<G> l = Lane<G>::x(i);
      xo[i] = (uint32_t)min(l.row, a.n - 1 - t0) * (uint32_t)a.x_stride * 2 + l.k * 2;
    }
#pragma unroll
    for (int i = 0; i < G::WLOADS; ++i) {
      const Lane<G> l = Lane<G>::w(i);
      wo[i] = (uint32_t)min(l.row, p.out - 1 - r0) * (uint32_t)(a.in / 8) * G::EIGHT + l.k / 8 * G::EIGHT;
    }
  }

  // Loads the stage of columns k0 ..; for columns past the last, which are not used, the first.
  __device__ __forceinline__ void stage(int k0, int in, AMK_LDS unsigned char* to) const {
    AMK_LDS unsigned char* dst = to + threadIdx.x / 64 * 1024;
    const bool whole = k0 + G::COLS <= in;
    const unsigned char *xs = x, *ws = w;
    uint32_t xi[G::XLOADS], wi[G::WLOADS];
#pragma unroll
    for (int i = 0; i < G::XLOADS; ++i) xi[i] = xo[i];
#pragma unroll
    for (int i = 0; i < G::WLOADS; ++i) wi[i] = wo[i];
    if (whole) {
      xs += (int64_t)k0 * 2;
      ws += (int64_t)(k0 / 8) * G::EIGHT;
    } else {
#pragma unroll
      for (int i = 0; i < G::XLOADS; ++i) {
        const int k = Lane<G>::x(i).k;
        xi[i] = xi[i] - k * 2 + (k0 + k < in ? k0 + k : 0) * 2;
      }
#pragma unroll
      for (int i = 0; i < G::WLOADS; ++i) {
        const int k = Lane<G>::w(i).k;
        wi[i] = wi[i] - k / 8 * G::EIGHT + (k0 + k < in ? k0 + k : 0) / 8 * G::EIGHT;
      }
    }
#pragma unroll
    for (int i = 0; i < G::XLOADS; ++i) load_lds16(xs + xi[i], dst + i * G::THREADS * 16);
#pragma unroll
    for (int i = 0; i < G::WLOADS; ++i) load_lds16(ws + wi[i], dst + (G::XCHUNKS + i * G::THREADS) * 16);
  }
};

// The products of this wave's share of the stage of columns k0 .., while the one that
// takes the place of the stage before (if more follow) is loaded into `next`.  xs, ws and
// next do not overlap: without that promise every read would wait for the loads.  TAIL:
// columns past the last count as 0.
template <int FMT, typename G, bool TAIL, bool GROUP32>
__device__ __forceinline__ void linear_step(const Source<G>& from, int in, int k0, bool more,
                                            const AMK_LDS unsigned char* __restrict__ xs,
                                            const AMK_LDS unsigned char* __restrict__ ws,
                                            AMK_LDS unsigned char* __restrict__ next, const float (&scale)[G::RB][2],
                                            f32x16 (&acc)[G::TB][G::RB]) {
  constexpr bool W4 = FMT == AMK_WEIGHTS_W4A16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
  const int kg = wave / (G::WT * G::WR), wt = wave % G::WT, wr = wave / G::WT % G::WR;
  const int kw = k0 + kg * G::BKW;  // the wave's first column
  if (more) from.stage(k0 + (G::STAGES - 1) * G::COLS, in, next);
  const int xrow = col % G::XR;  // few tokens: their rows repeat, and the results of the copies are left
  xs += (kg * G::XR + wt * 32 * G::TB + xrow) * G::XC * 16;
  ws += (kg * G::BR + wr * 32 * G::RB + col) * G::WC * 16;
  const bf16x8 nothing = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  constexpr int US = G::BKW / 32, SPAN = GROUP32 ? 1 : US;  // slices, and those of one group
  f32x16 part[G::TB][G::RB];  // W4A16: the sums of a group of columns
#pragma unroll
  for (int u = 0; u < US; ++u) {
    bf16x8 xf[G::TB][2], wf[G::RB][2];
#pragma unroll
    for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int c = (4 * u + 2 * half + s) ^ swizzle<G::XC>(32 * tb + xrow);
        xf[tb][s] = *(const AMK_LDS bf16x8*)(xs + 32 * tb * G::XC * 16 + c * 16);
        if (TAIL && kw + 32 * u + 16 * half + 8 * s >= in) xf[tb][s] = nothing;
      }
    if constexpr (W4)
      if (u % SPAN == 0)
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
          for (int rb = 0; rb < G::RB; ++rb) part[tb][rb] = f32x16{};
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
      if constexpr (TAIL && !W4)  // 0 times what lies there need not be 0
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (kw + 32 * u + 16 * half + 8 * s >= in) wf[rb][s] = nothing;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
        for (int rb = 0; rb < G::RB; ++rb) {
          f32x16& sum = W4 ? part[tb][rb] : acc[tb][rb];
          sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[tb][s], wf[rb][s], sum, 0, 0, 0);
        }
    if constexpr (W4) {
      // (columns past the last have no scale: 0 times a neighbour's need not be 0)
      if (u % SPAN == SPAN - 1 && !(TAIL && kw + 32 * (u - SPAN + 1) >= in)) {
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
          for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              acc[tb][rb][e] = __builtin_fmaf(scale[rb][u / SPAN], part[tb][rb][e], acc[tb][rb][e]);
      }
    }
  }
}

template <bool BF16, bool ADD>
__device__ __forceinline__ void put(void* to, int64_t at, float y) {
  if (BF16) {
    uint16_t* p = (uint16_t*)to + at;
    *p = f32_to_bf16(ADD ? bf16_to_f32(*p) + y : y);
  } else {
    float* p = (float*)to + at;
    *p = ADD ? *p + y : y;
  }
}

// Calls f with the kind of output as constants.
template <typename F>
__device__ __forceinline__ void by_output(const LinearArgs& a, F f) {
  if (a.y_bf16) a.accumulate ? f(std::true_type(), std::true_type()) : f(std::true_type(), std::false_type());
  else a.accumulate ? f(std::false_type(), std::true_type()) : f(std::false_type(), std::false_type());
}

// MANY: more than one matrix.  One alone is read straight from the arguments, since choosing
// costs its loads their early start (32 tokens int4 4096 -> 14336 13.9 us, chosen 14.5).
template <int FMT, typename G, bool GROUP32, bool MANY>
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
  // the row tiles of each matrix follow those of the one before
  int row_tile = tile / token_tiles;
  LinearPart part = a.part[0];
#pragma unroll
  for (int i = 1; i < (MANY ? 3 : 1); ++i) {
    const int before = (part.out + G::BR - 1) / G::BR;
    if (i < a.parts && row_tile >= before) {
      row_tile -= before;
      part = a.part[i];
    }
  }
  const int t0 = tile % token_tiles * G::BT, r0 = row_tile * G::BR;

  // under W4A16: this lane's rows of the scales, and the scales of its wave's next slice
  constexpr bool W4 = FMT == AMK_WEIGHTS_W4A16;
  const int groups = W4 ? a.in / a.group : 0, shift = W4 ? __builtin_ctz(a.group) : 0;
  const uint16_t* srow[G::RB];
  uint32_t ahead[G::RB][2];
#pragma unroll
  for (int rb = 0; rb < G::RB; ++rb)
    srow[rb] = (const uint16_t*)part.scale +
               (int64_t)min(r0 + (wr * G::RB + rb) * 32 + col, part.out - 1) * groups;
  auto fetch = [&](int k0) {
    if constexpr (W4)
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int u = 0; u < (GROUP32 ? G::BKW / 32 : 1); ++u)
          ahead[rb][u] = srow[rb][min((k0 + kg * G::BKW + 32 * u) >> shift, groups - 1)];
  };

  f32x16 acc[G::TB][G::RB] = {};
  const Source<G> from(a, part, t0, r0);
  constexpr int AHEAD = G::STAGES - 1;  // stages under way behind the one in use
  constexpr int LOADS = G::XLOADS + G::WLOADS;
  static_assert(!W4 || AHEAD == 1, "scales are fetched one stage ahead: waiting for them is waiting for all");
  fetch(0);
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i * G::COLS < a.in) from.stage(i * G::COLS, a.in, mem + i * G::STAGE);
  int k0 = 0, slot = 0;
  auto take = [&](auto tail) {
    // the stage is in once only the loads issued after its own are under way, and the
    // readers of the stage before are done
    if (k0 + AHEAD * G::COLS <= a.in) stage_barrier<(AHEAD - 1) * LOADS>();
    else stage_barrier<0>();
    float scale[G::RB][2] = {};
    if constexpr (W4) {
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb)
#pragma unroll
        for (int u = 0; u < (GROUP32 ? G::BKW / 32 : 1); ++u) {
          // with MANY the compiler converts a scale, and so waits for it, where it was loaded
          if constexpr (MANY) asm volatile("" : "+v"(ahead[rb][u]));
          scale[rb][u] = half_to_f32((uint16_t)ahead[rb][u]);
        }
    }
    fetch(k0 + G::COLS);
    AMK_LDS unsigned char *cur = mem + slot * G::STAGE, *next = mem + (slot ? slot - 1 : AHEAD) * G::STAGE;
    linear_step<FMT, G, decltype(tail)::value, GROUP32>(from, a.in, k0, k0 + AHEAD * G::COLS < a.in,
                                                        cur, cur + 16 * G::XCHUNKS, next, scale, acc);
    k0 += G::COLS;
    slot = slot == AHEAD ? 0 : slot + 1;
  };
  while (k0 + G::COLS <= a.in) take(std::false_type());
  if constexpr (!(W4 && !GROUP32 && G::KG == 1))  // else the columns are whole groups, and these whole stages
    if (k0 < a.in) take(std::true_type());

  if constexpr (G::KG == 1) {
    by_output(a, [&](auto bf16, auto add) {
#pragma unroll
      for (int rb = 0; rb < G::RB; ++rb) {
        const int r = r0 + (wr * G::RB + rb) * 32 + col;
        if (r >= part.out) continue;
        const float sc = FMT == AMK_WEIGHTS_W8A16 ? ((const float*)part.scale)[r] : 1.f;
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int t = t0 + (wt * G::TB + tb) * 32 + 8 * (e / 4) + 4 * half + e % 4;
            if (t < a.n) put<decltype(bf16)::value, decltype(add)::value>(part.y, t * a.y_stride + r, acc[tb][rb][e] * sc);
          }
      }
    });
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
        for (int e = 0; e < 16; ++e)
          sums[((kg * BLOCKS + tb * G::RB + rb) * 16 + e) * 64 + lane] = acc[tb][rb][e];
    __syncthreads();
    by_output(a, [&](auto bf16, auto add) {
#pragma unroll
      for (int n = 0; n < BLOCKS * 1024 / G::THREADS; ++n) {
        const int o = n * G::THREADS + threadIdx.x;
        const int l = o % 64, e = o / 64 % 16, rb = o / 1024 % G::RB, tb = o / 1024 / G::RB;
        const int t = t0 + tb * 32 + 8 * (e / 4) + 4 * (l / 32) + e % 4, r = r0 + rb * 32 + l % 32;
        if (t >= a.n || r >= part.out) continue;
        float y = sums[o];
#pragma unroll
        for (int g = 1; g < G::KG; ++g) y += sums[g * BLOCKS * 1024 + o];
        if (FMT == AMK_WEIGHTS_W8A16) y *= ((const float*)part.scale)[r];
        put<decltype(bf16)::value, decltype(add)::value>(part.y, t * a.y_stride + r, y);
      }
    });
  }
}

int64_t row_tiles(const LinearArgs& a, int rows) {
  int64_t tiles = 0;
  for (int i = 0; i < a.parts; ++i) tiles += (a.part[i].out + rows - 1) / rows;
  return tiles;
}

template <int FMT, typename G>
int launch_tile(const LinearArgs& a, hipStream_t st) {
  const int tt = (a.n + G::BT - 1) / G::BT, rt = (int)row_tiles(a, G::BR);
  const dim3 grid((unsigned)(((int64_t)tt * rt + 7) / 8 * 8));
  auto launch = [&](auto group32) {
    constexpr bool G32 = decltype(group32)::value;
    if (a.parts > 1) hipLaunchKernelGGL((linear_kernel<FMT, G, G32, true>), grid, dim3(G::THREADS), 0, st, a, tt, rt);
    else hipLaunchKernelGGL((linear_kernel<FMT, G, G32, false>), grid, dim3(G::THREADS), 0, st, a, tt, rt);
    return hipGetLastError() == hipSuccess ? AMK_OK : AMK_ERR_DEVICE;
  };
  if constexpr (FMT == AMK_WEIGHTS_W4A16 && G::BKW <= 64)
    if (a.group == 32) return launch(std::true_type());
  return launch(std::false_type());
}

template <int FMT>
int launch_fmt(const LinearArgs& a, hipStream_t st) {
  constexpr bool W4 = FMT == AMK_WEIGHTS_W4A16;
  const int64_t t32 = (int64_t)((a.n + 31) / 32) * row_tiles(a, 32);
  const int64_t t64 = (int64_t)((a.n + 63) / 64) * row_tiles(a, 64);
  const int64_t t128 = (int64_t)((a.n + 127) / 128) * row_tiles(a, 128);
  const int64_t t256 = (int64_t)((a.n + 255) / 256) * row_tiles(a, 256);
  // Few tokens, or too few tiles of 128 x 128: small tiles, their columns over 4 to 16 waves.
  // Stages of bf16 and int8 come in rings of three (30 tokens 14336 -> 4096 bf16 41 us, with two
  // 54); those of int4 wait for their scales (see linear_kernel), and where a CU takes one
  // tile, 16 waves on it hide some of that (30 tokens 14336 -> 4096 23.7 us, with 8 26.6).
  if (a.n <= 16) {  // x is padded to 16 only: 16 tokens bf16 4096 -> 4096 8.3 us, with 32 9.5
    if constexpr (W4)
      if (t32 <= 256) return launch_tile<FMT, Tile<FMT, 1, 1, 1, 1, 16, 64, 2, 16>>(a, st);
    return launch_tile<FMT, Tile<FMT, 1, 1, 1, 1, 8, W4 ? 64 : 32, W4 ? 2 : 3, 16>>(a, st);
  }
  // (17 tokens and more by some 33 000 rows of W have enough tiles of 128 x 128, most of whose
  // rows of x then repeat the last token: 4096 -> 128256 bf16 16 tokens 201 us, 17 202, 64 216;
  // int8 124, 178 and 193.)
  if (t128 < 256) {
    // One round of 32 x 32, two to a CU, where that takes them all, otherwise 64 x 64, which load
    // the same bytes in a round and half as many a product: 128 tokens int8 4096 -> 4096 13.0 us
    // in one round of 32 x 32 (20.5 in one of 64 x 64); 64 tokens bf16 4096 -> 14336 34.3 us in one
    // round of 64 x 64 (42.8 in two of 32 x 32).  Where CUs take two tiles of 32 x 32, 4 waves each
    // do (32 tokens int8 4096 -> 14336 13.8 us, with 8 14.9; one tile a CU, 4096 -> 8192, 10.0 and
    // 9.4), and bf16, whose stages are the largest, needs room for two tiles more than a third
    // stage (32 tokens 4096 -> 14336 27.1 us, with three 28.8).
    if (a.n <= 32 || t32 <= 512) {
      if (t32 <= 256) return launch_tile<FMT, Tile<FMT, 1, 1, 1, 1, W4 ? 16 : 8, W4 ? 64 : 32, W4 ? 2 : 3>>(a, st);
      return launch_tile<FMT, Tile<FMT, 1, 1, 1, 1, 4, 64, FMT == AMK_WEIGHTS_W8A16 ? 3 : 2>>(a, st);
    }
    // 64 x 64: 8 waves on one tile a CU, or 4 waves each on two.  300 tokens bf16 4096 -> 4096, 320
    // tiles, 26.4 us two to a CU (43.2 one); 200 tokens 14336 -> 4096, 256 tiles, 78 us one (104 two).
    if (t64 <= 256) return launch_tile<FMT, Tile<FMT, 2, 2, 1, 1, 8, W4 ? 64 : 32>>(a, st);
    return launch_tile<FMT, Tile<FMT, 2, 2, 1, 1, 4, W4 ? 64 : 32>>(a, st);
  }
  // the time of whole rounds of tiles: a 256 x 256 tile to a CU, or two of 128 x 128, which
  // take about 0.6 of its time together
  const int64_t large = (t256 + 255) / 256 * 10, medium = (t128 + 511) / 512 * 6;
  if constexpr (W4) {
    // where groups allow it, stages of 128 columns: half as many sums to scale, 2048 tokens
    // 4096 -> 14336 302 us (336 with stages of 64)
    if (a.group >= 128)
      return large <= medium ? launch_tile<FMT, Tile<FMT, 2, 2, 2, 4, 1, 128>>(a, st)
                             : launch_tile<FMT, Tile<FMT, 2, 2, 2, 2, 1, 128>>(a, st);
  }
  if (large <= medium) return launch_tile<FMT, Tile<FMT, W4 ? 2 : 4, 2, 2, 4, 1, 64>>(a, st);
  return launch_tile<FMT, Tile<FMT, 2, 2, 2, 2, 1, 64>>(a, st);
}

}  // namespace

int launch_linear(const LinearArgs& a, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (a.fmt == AMK_WEIGHTS_BF16) return launch_fmt<AMK_WEIGHTS_BF16>(a, st);
  if (a.fmt == AMK_WEIGHTS_W8A16) return launch_fmt<AMK_WEIGHTS_W8A16>(a, st);
  return launch_fmt<AMK_WEIGHTS_W4A16>(a, st);
}

}  // namespace amk
