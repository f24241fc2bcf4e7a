// Attention of several tokens: whole prompts (causal, packed sequences) and
// drafted trees over a KV cache.
//
// O = softmax(Q K^T scale) V per query head, in one pass over the keys with the
// running maximum m and sum l of each row: a tile of keys gives scores s, m' =
// max(m, max s), p = 2^(s - m') (scores in units of log2), l = l 2^(m - m') +
// sum p, O = O 2^(m - m') + p V, and O / l at the end.
//
// Rows.  The query heads of a KV group read the same K and V, so a workgroup's
// rows are (token, head of the group) pairs, row = token * group + head: K and V
// are staged once for all of them, and a causal tile of 128 rows spans few
// tokens, which leaves little masked work at the diagonal.
//
// Matrix cores.  Scores are taken transposed, S^T = K Q^T (32x32x16 bf16 tiles):
// a lane then holds keys of one query row, so the row's maximum and sum are
// taken within the lane and across one other lane.  The registers of S^T, rounded
// to bf16, are the B operand of O^T = V^T P^T as they lie, if the product's k slots
// 0..7 of lane half h stand for keys 4h..4h+3 and 8+4h..8+4h+3 of each 16: V^T's
// operand is read from the row-major tile in exactly that order by the
// transposed LDS reads.  P is rounded to bf16 (relative error at most 2^-8, of
// the size of the output's own rounding); l sums the unrounded p in fp32.  Taking P's
// remainder as a second operand brings an output's relative error from 0.0021 to 0.0017,
// all but that of its own rounding, for half as many products again: a prompt of 8192
// tokens 727 us, not 530, eight drafted tokens at 300 9.6, not 8.1.
//
// LDS.  K and V tiles are loaded straight to LDS (16 bytes a lane), two stages,
// so a tile's loads run under the previous tile's products.  Rows lie without
// padding, their 16-byte chunks permuted by the row so that neither the K reads
// (32 rows at one column) nor the transposed V reads (4 rows x 32 bytes) meet in
// a bank.
//
// Masked keys.  A score outside a row's keys is replaced, not added to, and p is then 0.
//
// Infinities and NaN of V.  0 * V is NaN there, and whether a small p is 0 depends on where
// the tiles begin.  A row whose O is not finite has its workgroup go through its tiles once
// more, with such values of V counted as 0, and adds them afterwards itself: those whose
// key it sees with any score but minus infinity, as their weight is then above 0 however
// small.  Rows that see none of them get the bits they have without them.
//
// What bounds it.  The two waves of a SIMD take turns at products and softmax: at a
// prompt of 8192 tokens, 32 query and 8 KV heads of 128, the matrix cores are busy 51%
// of the time and no LDS read meets another's bank: 535 us, 1030 TFLOP/s (a large bf16
// product reaches 1380).  Heads of 64 do half the products for the same softmax: six
// packed sequences of 4092 tokens, 32 and 4 heads, 50 us, 610 TFLOP/s.  64 drafted tokens
// at position 32001, 32 and 8 heads of 128, take 46 us and 8 more to join 32 splits (33
// MB of partial sums): 2.5 TB/s, where both the keys and the products have a floor of 24.
// Eight tokens at 300, 9 and 3 heads of 64, take 8.1 us, ten tiles one after another.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"

namespace amk {
namespace {

struct AttnArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;
  int32_t n_heads, n_kv, group;
  float scale2;       // scale * log2(e)
  int32_t splits, tiles;
  int32_t total_q, total_k;
  float* part_o;      // [splits][total_q * n_heads][head_dim], unnormalised
  float2* part_ml;    // [splits][total_q * n_heads] (m, l)
};

struct PromptArgs {
  const int32_t *cu_q, *cu_k;  // null: one sequence
  int32_t n_seqs;
};

struct TreeArgs {
  int32_t pos;
  TreeMasks masks;
};

// What one workgroup works on.
struct Span {
  int32_t q0, nq;     // queries of the sequence
  int32_t k0, nk;     // its keys
  int32_t tile;       // row tile within it; negative: none
};

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Row tile `tile` counted over all sequences: each wave looks at 64 sequences at
// a time and adds up their tiles.
__device__ Span find_span(const AttnArgs& a, const PromptArgs& p, int tile, int rows_per_tile) {
  if (!p.cu_q) return {0, a.total_q, 0, a.total_k, tile};
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < p.n_seqs; base += 64) {
    const int b = base + lane;
    Span s = {0, 0, 0, 0, -1};
    int mine = 0;
    if (b < p.n_seqs) {
      s.q0 = clamp_to(p.cu_q[b], 0, a.total_q);
      s.nq = clamp_to(p.cu_q[b + 1], s.q0, a.total_q) - s.q0;
      s.k0 = clamp_to(p.cu_k[b], 0, a.total_k);
      s.nk = clamp_to(p.cu_k[b + 1], s.k0, a.total_k) - s.k0;
      mine = (int)(((int64_t)s.nq * a.group + rows_per_tile - 1) / rows_per_tile);
    }
    int upto = mine;  // inclusive sum over the lanes
    for (int d = 1; d < 64; d <<= 1) {
      const int t = __shfl_up(upto, d);
      if (lane >= d) upto += t;
    }
    const uint64_t past = __ballot(tile < upto);
    if (past) {
      const int src = __ffsll((unsigned long long)past) - 1;
      s.tile = tile - (upto - mine);
      return {__shfl(s.q0, src), __shfl(s.nq, src), __shfl(s.k0, src), __shfl(s.nk, src), __shfl(s.tile, src)};
    }
    tile -= __shfl(upto, 63);
  }
  return {0, 0, 0, 0, -1};
}

__device__ __forceinline__ Span find_span(const AttnArgs& a, const TreeArgs& t, int tile, int) {
  return {0, a.total_q, 0, a.total_k, tile};
}

// The keys a row sees: all below `full`, and key full + j where bit j of `bits` is set.
struct Sees {
  int32_t full;
  uint64_t bits;
  // bit i: whether it sees key + i (0 <= i < 32), as far as key + i < end
  __device__ __forceinline__ uint32_t word(int key, int end) const {
    const int past = key - full;  // the first bit's place in `bits`
    uint64_t w = past <= -32 ? ~0ull : past < 0 ? bits << -past | ((1ull << -past) - 1) : past < 64 ? bits >> past : 0;
    const int room = end - key;
    if (room < 32) w &= room > 0 ? (1ull << room) - 1 : 0;
    return (uint32_t)w;
  }
};

__device__ __forceinline__ Sees sees_of(const PromptArgs&, const Span& s, int token) {
  return {max(0, s.nk - s.nq + token + 1), 0};
}
__device__ __forceinline__ Sees sees_of(const TreeArgs& t, const Span&, int token) {
  return {t.pos, t.masks.bits[token]};
}

// Keys the tokens up to `token` may see at all.
__device__ __forceinline__ int last_key(const PromptArgs&, const Span& s, int token) {
  return clamp_to(s.nk - s.nq + token + 1, 0, s.nk);
}
__device__ __forceinline__ int last_key(const TreeArgs&, const Span& s, int) { return s.nk; }

template <int HD>
__device__ __forceinline__ int k_swizzle(int row) {
  return HD == 128 ? row & 15 : (row >> 1) & 7;
}
template <int HD>
__device__ __forceinline__ int v_swizzle(int row) {
  return HD == 128 ? (row & 3) << 2 : (row & 2) << 1;
}

// Where a workgroup's tiles of K and V come from: the KV head's rows, and the bytes from a
// tile's first row to this lane's chunks.
template <int HD, int WAVES, int BN>
struct Source {
  static constexpr int CPR = HD / 8;                    // 16-byte chunks per row
  static constexpr int LOADS = BN * CPR / (64 * WAVES); // loads per lane and tile, of K and of V
  static constexpr int STEP = 64 * WAVES / CPR;         // rows from one load of a lane to its next
  static_assert(LOADS >= 1 && BN * CPR % (64 * WAVES) == 0, "whole loads");
  const unsigned char *k, *v;
  int64_t k_row, v_row;  // bytes
  int32_t nk;
  uint32_t ko[LOADS], vo[LOADS];

  static __device__ __forceinline__ uint32_t offset(int row, int64_t stride, int chunk) {
    return (uint32_t)row * (uint32_t)stride + chunk * 16;  // below 2^32: a row has at most 2^25 bytes
  }
  static __device__ __forceinline__ int k_chunk(int row) { return threadIdx.x % CPR ^ k_swizzle<HD>(row); }
  static __device__ __forceinline__ int v_chunk(int row) { return threadIdx.x % CPR ^ v_swizzle<HD>(row); }

  __device__ __forceinline__ Source(const uint16_t* k_, const uint16_t* v_, int64_t k_token, int64_t v_token, int nk_)
      : k((const unsigned char*)k_), v((const unsigned char*)v_), k_row(k_token * 2), v_row(v_token * 2), nk(nk_) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = i * STEP + threadIdx.x / CPR;
      ko[i] = offset(row, k_row, k_chunk(row));
      vo[i] = offset(row, v_row, v_chunk(row));
    }
  }

  // Loads tile t; rows past the last key repeat it: in range, and masked.
  __device__ __forceinline__ void tile(int t, AMK_LDS uint16_t* to) const {
    to += threadIdx.x / 64 * 512;
    const unsigned char *kt = k + (int64_t)(t * BN) * k_row, *vt = v + (int64_t)(t * BN) * v_row;
    uint32_t kc[LOADS], vc[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      kc[i] = ko[i];
      vc[i] = vo[i];
    }
    const int left = nk - 1 - t * BN;
    if (left < BN - 1) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = i * STEP + threadIdx.x / CPR;
        kc[i] = offset(min(row, left), k_row, k_chunk(row));
        vc[i] = offset(min(row, left), v_row, v_chunk(row));
      }
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      load_lds16(kt + kc[i], to + i * WAVES * 512);
      load_lds16(vt + vc[i], to + i * WAVES * 512 + BN * HD);
    }
  }
};

// The running result of this lane's query row: half of the columns of O, and m and l
// (l of the lane's own keys only).
template <int HD>
struct Running {
  f32x16 o[HD / 32];
  float m, l;
};

// Rows see all keys of a tile, or some only (PARTIAL); CLEAN: PARTIAL, and infinities and NaN
// of V count as 0.
enum class Keys { WHOLE, PARTIAL, CLEAN };

// Takes tile t, which lies in kt and vt, into the running result, while tile t + 1 (if
// more follow) is loaded into `next`.  kt, vt and next do not overlap: without that promise,
// which the compiler follows for pointers of few uses only, every read of tile t would wait
// for the loads of tile t + 1.  Returns whether (under CLEAN) this thread set values to 0.
template <int HD, int WAVES, int BN, Keys KEYS>
__device__ __forceinline__ bool attn_step(const Source<HD, WAVES, BN>& from, int t, bool more,
                                          const AMK_LDS uint16_t* __restrict__ kt,
                                          AMK_LDS uint16_t* __restrict__ vt, AMK_LDS uint16_t* __restrict__ next,
                                          const bf16x8* q, const Sees& sees, int kend, float scale2,
                                          Running<HD>& run) {
  constexpr int KB = BN / 32, DB = HD / 32;
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  if (more) from.tile(t + 1, next);

  f32x16 sc[KB] = {};
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      const int r = kb * 32 + col;
      const bf16x8 kf = *(const AMK_LDS bf16x8*)(kt + r * HD + ((2 * i + half) ^ k_swizzle<HD>(r)) * 8);
      sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[i], sc[kb], 0, 0, 0);
    }

  if constexpr (KEYS == Keys::WHOLE) {
    // K's operands are read four ahead of the products that take them (0x100: LDS reads, 8:
    // matrix instructions)
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < KB * HD / 16 - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
  }

  if constexpr (KEYS != Keys::WHOLE) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const uint32_t word = sees.word(t * BN + kb * 32, kend) >> 4 * half;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(word >> (8 * (i / 4) + i % 4) & 1)) sc[kb][i] = -INFINITY;
    }
  }

  float top = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[kb][i]);
  top = fmaxf(top, __shfl_xor(top, 32));
  // m follows the maximum only where a score exceeds it by 2^8: sums and products lose
  // nothing by weights of up to 256, and most tiles need not rescale O.  Each row goes by
  // its own scores: what another row of the wave sees does not move its m
  const float high = top * scale2;
  const bool moves = high > run.m + 8.f;
  if (__any(moves)) {
    const float m = moves ? high : run.m;
    const float keep = moves ? __builtin_amdgcn_exp2f(run.m - m) : 1.f;
    run.m = m;
    run.l *= keep;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) run.o[d][i] *= keep;
  }
  const float base = run.m == -INFINITY ? 0.f : run.m;  // nothing seen yet: p = 2^-inf = 0
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kb][i], scale2, -base));
      run.l += sc[kb][i];
    }

  bool odd = false;
  if constexpr (KEYS == Keys::CLEAN) {
#pragma unroll
    for (int i = 0; i < Source<HD, WAVES, BN>::LOADS; ++i) {
      AMK_LDS u32x4* at = (AMK_LDS u32x4*)vt + i * 64 * WAVES + threadIdx.x;
      u32x4 x = *at;
      bool here = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool lo = (x[e] & 0x7f80u) == 0x7f80u, hi = (x[e] & 0x7f800000u) == 0x7f800000u;
        here |= lo | hi;
        x[e] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
      }
      if (here) *at = x;
      odd |= here;
    }
    __syncthreads();
  }

  bf16x8 p[KB][2];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) p[kb][i / 8][i % 8] = (__bf16)sc[kb][i];
  const int vr = 4 * half + (lane & 15) / 4;  // + multiples of 8
  const int vc = ((lane >> 4) & 1) * 2 + (lane & 3) / 2, ve = (lane & 1) * 4;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const AMK_LDS uint16_t* at = vt + (kb * 32 + ks * 16 + vr) * HD + ((4 * d + vc) ^ v_swizzle<HD>(vr)) * 8 + ve;
        const s16x4 lo = read_tr16(at), hi = read_tr16(at + 8 * HD);
        const s16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        run.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), p[kb][ks], run.o[d], 0, 0, 0);
      }
  return odd;
}

// Adds the infinities and NaN of V at keys [key, end) to the rows that see their key with a
// score other than minus infinity.  Rare: a lane takes its row's key by key.
template <int HD, typename Source>
__device__ __forceinline__ void add_odd(const Source& from, int key, int end, const bf16x8* q, const Sees& sees,
                                        int half, Running<HD>& run) {
  for (; key < end; ++key) {
    const unsigned char* kp = from.k + key * from.k_row + half * 16;
    float score = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      const u32x4 a = __builtin_bit_cast(u32x4, q[i]), b = *(const u32x4*)(kp + 32 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t qw = a[e], kw = b[e];
        score = __builtin_fmaf(bf16_to_f32((uint16_t)qw), bf16_to_f32((uint16_t)kw), score);
        score = __builtin_fmaf(bf16_to_f32((uint16_t)(qw >> 16)), bf16_to_f32((uint16_t)(kw >> 16)), score);
      }
    }
    score += __shfl_xor(score, 32);
    if (!(sees.word(key, end) & 1) || score == -INFINITY) continue;
    const uint16_t* vp = (const uint16_t*)(from.v + key * from.v_row) + 4 * half;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 w = *(const u32x2*)(vp + 32 * d + 8 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t word = w[e / 2];
          const float x = bf16_to_f32((uint16_t)(word >> e % 2 * 16));
          if (!(fabsf(x) < INFINITY)) run.o[d][4 * i + e] += x;
        }
      }
  }
}

template <int HD, int WAVES, int BN, typename Which>
__global__ void __launch_bounds__(64 * WAVES, 2) attn_kernel(const AttnArgs a, const Which w) {
  constexpr int ROWS = 32 * WAVES, DB = HD / 32;
  constexpr int TILE = BN * HD;  // elements of a K or V tile
  // two stages of K and V and a note of what is rare: one variable, since the compiler keeps
  // what it knows of attn_step's pointers only where a kernel has no second one
  __shared__ __align__(16) uint16_t lds[4 * TILE + 8];
  AMK_LDS uint16_t* stages = (AMK_LDS uint16_t*)lds;
  // [0] a row is not finite; V's infinities and NaN lie in tiles [1] .. below [2]
  AMK_LDS int* note = (AMK_LDS int*)(stages + 4 * TILE);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int half = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.x % a.n_kv;
  const int rest = blockIdx.x / a.n_kv;
  const int split = rest % a.splits;
  // later tiles of a causal prompt have more keys: the last ones start first
  const Span s = find_span(a, w, a.tiles - 1 - rest / a.splits, ROWS);
  if (s.tile < 0) return;
  const int rows = s.nq * a.group, row0 = s.tile * ROWS;
  if (row0 >= rows) return;
  const int last_row = min(rows, row0 + ROWS) - 1;

  const int row = row0 + wave * 32 + col;
  const bool valid = row <= last_row;
  const int token = valid ? row / a.group : 0, head = valid ? kvh * a.group + row % a.group : 0;
  Sees sees = {0, 0};
  if (valid) sees = sees_of(w, s, token);
  const int kend = last_key(w, s, last_row / a.group);
  const int kfull = min(sees_of(w, s, row0 / a.group).full, kend);  // seen by every row of the tile

  bf16x8 q[HD / 16];
  {
    const uint16_t* qp = a.q + (s.q0 + token) * a.q_token + head * a.q_head + half * 8;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      u32x4 v = {0, 0, 0, 0};
      if (valid) v = *(const u32x4*)(qp + 16 * i);
      q[i] = __builtin_bit_cast(bf16x8, v);
    }
  }

  const int ktiles = (kend + BN - 1) / BN;
  const int t0 = (int)((int64_t)ktiles * split / a.splits), t1 = (int)((int64_t)ktiles * (split + 1) / a.splits);
  const int tf = max(t0, min(t1, kfull / BN));  // tiles that every row sees whole
  const Source<HD, WAVES, BN> from(a.k + s.k0 * a.k_token + kvh * a.k_head, a.v + s.k0 * a.v_token + kvh * a.v_head,
                                   a.k_token, a.v_token, s.nk);
  if (threadIdx.x == 0) {
    note[0] = 0;
    note[1] = t1;
    note[2] = t0;
  }
  Running<HD> run;
  auto pass = [&](auto keys) {
    constexpr Keys KEYS = decltype(keys)::value;
    run = {};
    run.m = -INFINITY;
    int first = t1, past = t0, t = t0, stage = 0;  // tiles in which this thread set values of V to 0
    if (t0 < t1) from.tile(t0, stages);
    if constexpr (KEYS == Keys::PARTIAL)
      for (; t < tf; ++t, stage ^= 1) {
        stage_barrier<0>();  // tile t is in, and the readers of the other stage are done
        AMK_LDS uint16_t* cur = stages + stage * 2 * TILE;
        attn_step<HD, WAVES, BN, Keys::WHOLE>(from, t, t + 1 < t1, cur, cur + TILE, stages + (stage ^ 1) * 2 * TILE, q,
                                              sees, kend, a.scale2, run);
      }
    for (; t < t1; ++t, stage ^= 1) {
      stage_barrier<0>();
      AMK_LDS uint16_t* cur = stages + stage * 2 * TILE;
      const bool odd = attn_step<HD, WAVES, BN, KEYS>(from, t, t + 1 < t1, cur, cur + TILE,
                                                      stages + (stage ^ 1) * 2 * TILE, q, sees, kend, a.scale2, run);
      if (KEYS == Keys::CLEAN && odd) {
        first = min(first, t);
        past = t + 1;
      }
    }
    if (KEYS == Keys::CLEAN && first < past) {
      __hip_atomic_fetch_min(note + 1, first, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      __hip_atomic_fetch_max(note + 2, past, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
  };
  pass(std::integral_constant<Keys, Keys::PARTIAL>());
  float l = run.l + __shfl_xor(run.l, 32);
  float zero = 0.f;  // NaN if O holds an infinity or NaN
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(run.o[d][i], 0.f, zero);
  // a row whose sum is NaN stays NaN
  if (valid && l == l && zero != zero) note[0] = 1;
  __syncthreads();
  if (note[0]) {
    pass(std::integral_constant<Keys, Keys::CLEAN>());
    l = run.l + __shfl_xor(run.l, 32);
    __syncthreads();
    add_odd<HD>(from, note[1] * BN, min(note[2] * BN, kend), q, sees, half, run);
  }

  if (!valid) return;
  if (a.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* op = a.out + (s.q0 + token) * a.out_token + head * a.out_head + 4 * half;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 v = {pack_bf16(run.o[d][4 * i] * inv, run.o[d][4 * i + 1] * inv),
                         pack_bf16(run.o[d][4 * i + 2] * inv, run.o[d][4 * i + 3] * inv)};
        *(u32x2*)(op + 32 * d + 8 * i) = v;
      }
  } else {
    const int64_t at = ((int64_t)split * a.total_q + s.q0 + token) * a.n_heads + head;
    if (half == 0) a.part_ml[at] = make_float2(run.m, l);
    float* op = a.part_o + at * HD + 4 * half;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 v = {run.o[d][4 * i], run.o[d][4 * i + 1], run.o[d][4 * i + 2], run.o[d][4 * i + 3]};
        *(f32x4*)(op + 32 * d + 8 * i) = v;
      }
  }
}

// Joins the splits of each (token, head), one wave each: HD / 4 lanes take a split's row
// of O, so 2 or 4 splits are read side by side and 8 or 16 are on their way.  Splits
// that saw nothing for the row (l = 0) are left out; the infinities and NaN of any other
// stay, also where its weight is too small for fp32.
template <int HD>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnArgs a, const int32_t* cu_q, int32_t n_seqs) {
  constexpr int LANES = HD / 4, SIDE = 64 / LANES, AHEAD = 4;
  const int lane = threadIdx.x & 63, sub = lane / LANES;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), all = (int64_t)a.total_q * a.n_heads;
  if (at >= all) return;
  const int64_t token = at / a.n_heads;
  const int head = (int)(at % a.n_heads);
  if (cu_q && (token < cu_q[0] || token >= cu_q[n_seqs])) return;
  float m = -INFINITY;
  for (int i = lane; i < a.splits; i += 64) m = fmaxf(m, a.part_ml[i * all + at].x);
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  const float base = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const float* po = a.part_o + at * HD + lane % LANES * 4;
  for (int i0 = 0; i0 < a.splits; i0 += 64) {
    float f = -1.f;  // left out
    if (i0 + lane < a.splits) {
      const float2 ml = a.part_ml[(i0 + lane) * all + at];
      if (ml.y != 0.f) {
        f = __builtin_amdgcn_exp2f(ml.x - base);
        l += f * ml.y;
      }
    }
    const int n = min(64, a.splits - i0);
    for (int i = 0; i < n; i += SIDE * AHEAD) {
      f32x4 v[AHEAD];
      float w[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int k = i + u * SIDE + sub;
        w[u] = __shfl(f, k & 63);
        if (k >= n) w[u] = -1.f;
        v[u] = *(const f32x4*)(po + (int64_t)(i0 + min(k, n - 1)) * all * HD);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (w[u] > 0.f) o += w[u] * v[u];
        else if (w[u] == 0.f)
          for (int e = 0; e < 4; ++e)
            if (!(fabsf(v[u][e]) < INFINITY)) o[e] += v[u][e];
    }
  }
  for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    for (int d = 32; d >= LANES; d >>= 1) o[e] += __shfl_xor(o[e], d);
  if (sub) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const u32x2 r = {pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  *(u32x2*)(a.out + token * a.out_token + head * a.out_head + lane * 4) = r;
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

AttnPlan with_workspace(AttnPlan p, int n_heads, int head_dim, int total_q) {
  const size_t rows = (size_t)p.splits * total_q * n_heads;
  p.workspace = p.splits == 1 ? 0 : up256(rows * head_dim * sizeof(float)) + rows * sizeof(float2);
  return p;
}

// Workgroups a plan with splits may launch: eight waves a CU, two per SIMD.  That is what
// runs at once for heads of 128 in workgroups of 2 waves and more.  Workgroups of one wave have
// LDS for four a CU, so the longest contexts of a few tokens take two rounds; heads of 64
// would leave room for 9 to 12 waves.
int resident(int waves) { return 256 * 8 / waves; }

// Waves (32 rows each) of a workgroup.  Eight share a tile of K and V among twice the rows
// of four, but mask more at a causal diagonal, and `many` says that this pays: heads of 128,
// us with eight / four waves, 32 and 8 heads: one prompt of 8192 tokens 523 / 540, one of 4096
// 148 / 161, two of 2048 85 / 90, two of 1800 71 / 72, three of 1400 79 / 72, four of 1024 66 / 59;
// a tree of 64 tokens at 32001 54 / 59.  Prompts take eight from 8192 rows of a sequence on.
// One KV head has too few tiles for it (8 and 1 heads, three of 1500 tokens 49 / 39).  Heads
// of 64 gain nothing (a prompt of 8192 330 / 318).
int waves_for(int64_t rows, int head_dim, bool many) {
  return rows <= 32 ? 1 : rows <= 64 ? 2 : many && head_dim == 128 ? 8 : 4;
}

AttnArgs make_args(const amk_attention_t& a, const AttnPlan& p, int total_q, int total_k, void* workspace) {
  AttnArgs r;
  r.q = (const uint16_t*)a.q; r.k = (const uint16_t*)a.k; r.v = (const uint16_t*)a.v; r.out = (uint16_t*)a.out;
  r.q_token = a.q_token; r.q_head = a.q_head; r.k_token = a.k_token; r.k_head = a.k_head;
  r.v_token = a.v_token; r.v_head = a.v_head; r.out_token = a.out_token; r.out_head = a.out_head;
  r.n_heads = a.n_heads; r.n_kv = a.n_kv_heads; r.group = a.n_heads / a.n_kv_heads;
  r.scale2 = (float)((double)a.scale * 1.4426950408889634);
  r.splits = p.splits; r.tiles = p.tiles; r.total_q = total_q; r.total_k = total_k;
  r.part_o = (float*)workspace;
  r.part_ml = (float2*)((char*)workspace + up256((size_t)p.splits * total_q * a.n_heads * a.head_dim * sizeof(float)));
  return r;
}

template <int HD, typename Which>
void launch_hd(const AttnArgs& r, const AttnPlan& p, const Which& w, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)p.tiles * p.splits * r.n_kv));
  if (p.waves == 1) hipLaunchKernelGGL((attn_kernel<HD, 1, 32, Which>), grid, dim3(64), 0, st, r, w);
  else if (p.waves == 2) hipLaunchKernelGGL((attn_kernel<HD, 2, 32, Which>), grid, dim3(128), 0, st, r, w);
  else if (p.waves == 4) hipLaunchKernelGGL((attn_kernel<HD, 4, 64, Which>), grid, dim3(256), 0, st, r, w);
  else if constexpr (HD == 128) hipLaunchKernelGGL((attn_kernel<HD, 8, 64, Which>), grid, dim3(512), 0, st, r, w);
}

template <typename Which>
int launch_attn(const AttnArgs& r, const AttnPlan& p, int head_dim, const Which& w, const int32_t* cu_q, int n_seqs,
                hipStream_t st) {
  if (head_dim == 128) launch_hd<128>(r, p, w, st);
  else launch_hd<64>(r, p, w, st);
  if (hipGetLastError() != hipSuccess) return AMK_ERR_DEVICE;
  if (p.splits > 1) {
    const dim3 grid((unsigned)(((int64_t)r.total_q * r.n_heads + 3) / 4));
    if (head_dim == 128) hipLaunchKernelGGL(attn_join_kernel<128>, grid, dim3(256), 0, st, r, cu_q, n_seqs);
    else hipLaunchKernelGGL(attn_join_kernel<64>, grid, dim3(256), 0, st, r, cu_q, n_seqs);
    if (hipGetLastError() != hipSuccess) return AMK_ERR_DEVICE;
  }
  return AMK_OK;
}

}  // namespace

// Splits of the keys: as many workgroups as run at once, if every one has `least` keys.
int splits_for(int64_t blocks, int waves, int64_t keys, int least) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(resident(waves) / blocks, (keys + least - 1) / least));
}

AttnPlan prompt_plan(int n_heads, int n_kv_heads, int head_dim, int n_seqs, int total_q, int total_k) {
  AttnPlan p;
  const int64_t rows = (int64_t)total_q * (n_heads / n_kv_heads);
  p.waves = waves_for(rows, head_dim, rows / n_seqs >= 8192);
  // whole tiles of the sum, and one that is not whole per sequence
  p.tiles = (int)(rows / (32 * p.waves) + std::min<int64_t>(n_seqs, rows));
  p.splits = splits_for((int64_t)p.tiles * n_kv_heads, p.waves, total_k, 256);
  return with_workspace(p, n_heads, head_dim, total_q);
}

AttnPlan tree_plan(int n_heads, int n_kv_heads, int head_dim, int n, int pos) {
  AttnPlan p;
  const int64_t rows = (int64_t)n * (n_heads / n_kv_heads);
  p.waves = waves_for(rows, head_dim, rows > 128);
  p.tiles = (int)((rows + 32 * p.waves - 1) / (32 * p.waves));
  // Up to 320 keys whole, beyond in ranges of 128, which need the join.  us whole / split of 8
  // tokens, 9 and 3 heads of 64: 200 keys 6.7 / 8.4, 260 7.9 / 8.1, 320 8.3 / 8.4, 400 9.8 / 8.4;
  // of 16, 32 and 4 heads of 64: 320 keys 8.7 / 9.3, 400 10.6 / 9.3.  The tiles of wider heads take
  // longer, and pay from fewer keys on: 8 tokens, 32 and 8 heads of 128, 200 keys 10.2 / 10.6, 260
  // 12.0 / 10.0, 320 12.7 / 10.7.
  const int64_t keys = (int64_t)pos + n;
  p.splits = keys <= 320 ? 1 : splits_for((int64_t)p.tiles * n_kv_heads, p.waves, keys, 128);
  return with_workspace(p, n_heads, head_dim, n);
}

size_t attention_workspace_most(int n_heads, int n_kv_heads, int head_dim) {
  // a plan with splits has at most resident(waves) workgroups of 32 * waves rows
  const size_t rows = (size_t)resident(1) * 32;
  return up256(rows * head_dim * sizeof(float)) + rows * sizeof(float2);
}

int launch_prompt(const amk_attention_t& a, const AttnPlan& p, const int32_t* cu_q, const int32_t* cu_k, int n_seqs,
                  int total_q, int total_k, void* workspace, void* stream) {
  return launch_attn(make_args(a, p, total_q, total_k, workspace), p, a.head_dim, PromptArgs{cu_q, cu_k, n_seqs}, cu_q,
                     n_seqs, (hipStream_t)stream);
}

int launch_tree(const amk_attention_t& a, const AttnPlan& p, int n, int pos, const TreeMasks& m, void* workspace,
                void* stream) {
  return launch_attn(make_args(a, p, n, pos + n, workspace), p, a.head_dim, TreeArgs{pos, m}, nullptr, 0,
                     (hipStream_t)stream);
}

}  // namespace amk
