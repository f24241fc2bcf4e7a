// Log probabilities of given tokens, entropy and the most probable alternatives
// of rows of logits.
//
// With m the row's maximum, s = sum e^(x - m) and u = sum (x - m) e^(x - m):
// log p(x) = x - m - log s and H = log s - u / s.  A workgroup takes a chunk of a
// row into registers in one read and leaves (m, s, u) and the chunk's best
// entries; a second kernel, one workgroup a row, joins the chunks.  One read of
// the logits is all that cannot be avoided, so HBM and the vector ALUs (some 28
// instructions an entry) bound large calls and the two launches small ones.
// Chunks of 8192 entries are few for the join and leave registers for six waves
// per SIMD: 1024 x 128256 fp32 logits with 20 alternatives take 99 us (5.3 TB/s),
// with five waves 106; bf16 104.  (At six, one register of the fp32 kernel spills, 8 bytes a
// lane.)  Quarter chunks for few rows only make the join longer: one row 12.6 us and 16 rows
// 30.5, not 8.8 and 13.9.
//
// Best entries.  Each lane's maximum over the workgroup's waves gives 64 maxima
// of disjoint groups; the top-th largest of them is a value that at least `top`
// entries reach, and few more do unless many are equal.  The entries that reach
// it are listed and ranked by counting.  Where they overflow the list (rows of
// few distinct values), `top` rounds each find the best entry after the last.
// An entry is a 64-bit key, the value's order above the inverted index, so that
// larger keys come first and equal values by the lower index: the result is the
// same however the list was filled.
#include <algorithm>
#include <cmath>

#include "ops.h"
#include "ops_device.h"

namespace amk {
namespace {

constexpr int NT = 256, WAVES = NT / 64;
constexpr int PER = 32;     // entries of a thread: a chunk is 8192 entries
constexpr int NJ = 256;     // threads of the joining kernel
constexpr int LIST = 1024;  // keys ranked by counting
constexpr int SEG = LIST / WAVES;  // of them, one wave's

typedef unsigned long long Key;  // 0: none

__device__ __forceinline__ Key key_of(float x, int i) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);  // one zero
  const uint32_t order = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (Key)order << 32 | (uint32_t)~i;
}
__device__ __forceinline__ int index_of(Key k) { return ~(int)(uint32_t)k; }
__device__ __forceinline__ float value_of(Key k) {
  const uint32_t order = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, order & 0x80000000u ? order & 0x7fffffffu : ~order);
}

template <int TYPE>
struct Elem;
template <>
struct Elem<AMK_F32> {
  typedef float T;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float bits(uint32_t v) { return __builtin_bit_cast(float, v); }
};
template <>
struct Elem<AMK_BF16> {
  typedef uint16_t T;
  static __device__ __forceinline__ float get(uint16_t v) { return bf16_to_f32(v); }
  static __device__ __forceinline__ float bits(uint32_t v) { return get((uint16_t)v); }
};
template <>
struct Elem<AMK_F16> {
  typedef uint16_t T;
  static __device__ __forceinline__ float get(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ __forceinline__ float bits(uint32_t v) { return get((uint16_t)v); }
};

__device__ __forceinline__ Key best_of_wave(Key v) {
  for (int d = 32; d; d >>= 1) v = max(v, (Key)__shfl_xor(v, d));
  return v;
}

__device__ __forceinline__ Key least_of_wave(Key v) {
  for (int d = 32; d; d >>= 1) v = min(v, (Key)__shfl_xor(v, d));
  return v;
}

// Maximum and sums of one chunk; s is NaN where the chunk holds a NaN or plus infinity.
struct ChunkStat {
  float m, s, u;
};

template <int TYPE>
__global__ void __launch_bounds__(NT, 6) logprob_chunk_kernel(const typename Elem<TYPE>::T* logits, int64_t row_stride,
                                                              int vocab, int chunks, int top, ChunkStat* stats,
                                                              Key* best) {
  typedef typename Elem<TYPE>::T T;
  constexpr int VEC = 16 / sizeof(T);
  __shared__ float lane_max[WAVES][64];
  __shared__ float2 sums[WAVES];
  __shared__ Key list[WAVES][SEG];
  __shared__ int counts[WAVES];
  __shared__ int exceeds[WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const T* p = logits + (int64_t)row * row_stride;
  // chunks are cut at 16-byte boundaries of memory: `skew` entries before the row
  const int skew = (int)(((uintptr_t)p & 15) / sizeof(T));
  const int first = chunk * (NT * PER) - skew + (int)threadIdx.x * VEC;  // entry of x[0]
  auto entry = [&](int j) { return first + j / VEC * (NT * VEC) + j % VEC; };

  float x[PER];
#pragma unroll
  for (int j = 0; j < PER; j += VEC) {
    const int i = entry(j);
    if (i >= 0 && i + VEC <= vocab) {
      const u32x4 v = __builtin_nontemporal_load((const u32x4*)(p + i));
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const uint32_t word = v[sizeof(T) == 4 ? e % 4 : e / 2 % 4];
        x[j + e] = Elem<TYPE>::bits(sizeof(T) == 4 ? word : word >> (e % 2 * 16));
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[j + e] = i + e >= 0 && i + e < vocab ? Elem<TYPE>::get(p[i + e]) : -INFINITY;
    }
  }
  // maxima of four entries each, then of all of the lane's (NaN left out)
  float four[PER / 4], mine;
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) {
    four[j] = fmaxf(fmaxf(x[4 * j], x[4 * j + 1]), fmaxf(x[4 * j + 2], x[4 * j + 3]));
    mine = j ? fmaxf(mine, four[j]) : four[j];
  }
  lane_max[wave][lane] = mine;
  __syncthreads();
  float group = lane_max[0][lane];  // of this lane in all waves
#pragma unroll
  for (int i = 1; i < WAVES; ++i) group = fmaxf(group, lane_max[i][lane]);
  const float m = wave_max(group);
  if (top) {  // how many of the 64 exceed this lane's, a share of them counted by each wave
    int more = 0;
#pragma unroll
    for (int o = 0; o < 64 / WAVES; ++o)
      more += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, group),
                                                                  wave * (64 / WAVES) + o)) > group;
    exceeds[wave][lane] = more;
  }
  // a NaN makes s NaN, and so does plus infinity (its own difference from m)
  const float base = m == -INFINITY ? 0.f : m;
  float s = 0.f, u = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const float z = x[j] - base, e = __expf(z);
    s += e;
    u += fmaxf(z, -200.f) * e;  // e is 0 long before
  }
  s = wave_sum(s);
  u = wave_sum(u);
  if (lane == 0) sums[wave] = make_float2(s, u);
  __syncthreads();
  if (threadIdx.x == 0) {
    s = sums[0].x;
    u = sums[0].y;
    for (int i = 1; i < WAVES; ++i) {
      s += sums[i].x;
      u += sums[i].y;
    }
    stats[blockIdx.x] = {m, s, u};
  }
  if (top == 0) return;

  Key* to = best + (int64_t)blockIdx.x * top;
  // the top-th largest of the 64: the least that fewer than `top` exceed
  int more = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) more += exceeds[w][lane];
  const float least = -wave_max(more < top ? -group : -INFINITY);
  const bool inside = least > -INFINITY;  // entries outside the row are minus infinity
  int count = 0;                          // of the wave, in its own segment
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) {
    if (!__any(four[j] >= least)) continue;
#pragma unroll
    for (int e = 4 * j; e < 4 * j + 4; ++e) {
      const int i = entry(e);
      const bool in = x[e] >= least && (inside || (i >= 0 && i < vocab));
      const uint64_t lanes = __ballot(in);
      if (!lanes) continue;
      const int at = count + __popcll(lanes & ((1ull << lane) - 1));
      if (in && at < SEG) list[wave][at] = key_of(x[e], i);
      count += __popcll(lanes);
    }
  }
  if (lane == 0) counts[wave] = count;
  __syncthreads();
  int most = 0, all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    most = max(most, counts[w]);
    all += counts[w];
  }
  if (all <= 64) {  // the usual case: one wave ranks them from its registers
    if (wave) return;
    int w = 0, at = lane;  // this lane's key: the at-th of segment w
#pragma unroll
    for (int i = 0; i + 1 < WAVES; ++i)
      if (w == i && at >= counts[i]) {
        at -= counts[i];
        ++w;
      }
    const Key k = lane < all ? list[w][at] : 0;
    int rank = 0;
    for (int o = 0; o < all; ++o) {
      const Key other = (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), o) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane((int)k, o);
      rank += other > k;
    }
    if (lane < all && rank < top) to[rank] = k;
    if (lane >= all && lane < top) to[lane] = 0;
    return;
  }
  if (most <= SEG) {
    for (int c = lane; c < count; c += 64) {  // each wave ranks its own keys
      const Key k = list[wave][c];
      int rank = 0;
      for (int w = 0; w < WAVES; ++w)
        for (int o = 0; o < counts[w]; ++o) rank += list[w][o] > k;
      if (rank < top) to[rank] = k;
    }
    return;
  }
  Key last = ~0ull;
  for (int r = 0; r < top; ++r) {
    Key k = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = entry(j);
      const Key c = key_of(x[j], i);
      if (i >= 0 && i < vocab && x[j] == x[j] && c < last) k = max(k, c);
    }
    k = best_of_wave(k);
    __syncthreads();
    if (lane == 0) list[wave][0] = k;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) k = max(k, list[w][0]);
    if (threadIdx.x == 0) to[r] = k;
    last = k;
  }
}

template <int TYPE>
__global__ void __launch_bounds__(NJ) logprob_join_kernel(const typename Elem<TYPE>::T* logits, int64_t row_stride,
                                                          int vocab, int chunks, int top, const ChunkStat* stats,
                                                          const Key* best, const int32_t* tokens, float* logprob,
                                                          float* entropy, int32_t* top_ids, float* top_logprobs) {
  __shared__ Key list[LIST];
  __shared__ int count;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const Key* from = best + (int64_t)row * chunks * top;
  if (threadIdx.x == 0) count = 0;

  // every wave joins the statistics by itself
  const ChunkStat* st = stats + (int64_t)row * chunks;
  float m = -INFINITY;
  for (int c = lane; c < chunks; c += 64) m = fmaxf(m, st[c].m);
  m = wave_max(m);
  float s = 0.f, u = 0.f;
  for (int c = lane; c < chunks; c += 64) {
    // a chunk's sums move to the row's maximum: x - m = (x - mc) + (mc - m)
    const ChunkStat k = st[c];
    const bool none = k.m == -INFINITY && k.s == 0.f;
    const float d = none ? 0.f : fmaxf(k.m - m, -200.f), f = __expf(d);
    s += k.s * f;
    u += (k.u + d * k.s) * f;
  }
  s = wave_sum(s);
  u = wave_sum(u);
  const bool bad = !(s < INFINITY) || m == -INFINITY;  // NaN, plus infinity or nothing possible
  const float ls = logf(s), none = __builtin_nanf("");
  if (threadIdx.x == 0) {
    if (entropy) entropy[row] = bad ? none : ls - u / s;
    if (tokens) {
      const int t = tokens[row];
      float lp = none;
      if (!bad && t >= 0 && t < vocab) lp = Elem<TYPE>::get(logits[row * row_stride + t]) - m - ls;
      logprob[row] = lp;
    }
  }
  if (top == 0) return;

  // The chunks' lists are in order, so the first q of each make `top` keys that are at
  // least the least of their q-th: keys below that are out, and few are left to rank.
  const int q = (top + chunks - 1) / chunks;
  Key least = ~0ull;
  for (int c = lane; c < chunks; c += 64) least = min(least, from[c * top + q - 1]);
  least = least_of_wave(least);
  __syncthreads();
  const int keys = chunks * top;
  for (int i = threadIdx.x; i < keys; i += NJ) {
    const Key k = from[i];
    if (k && k >= least) {
      const int at = atomicAdd(&count, 1);
      if (at < LIST) list[at] = k;
    }
  }
  __syncthreads();
  const int listed = count;
  auto put = [&](int r, Key k) {
    top_ids[(int64_t)row * top + r] = bad || !k ? -1 : index_of(k);
    top_logprobs[(int64_t)row * top + r] = bad || !k ? none : value_of(k) - m - ls;
  };
  if (listed <= LIST) {
    for (int c = threadIdx.x; c < listed; c += NJ) {
      const Key k = list[c];
      int rank = 0;
#pragma unroll 4
      for (int o = 0; o < listed; ++o) rank += list[o] > k;
      if (rank < top) put(rank, k);
    }
    for (int r = listed + threadIdx.x; r < top; r += NJ) put(r, 0);
    return;
  }
  // too many equal candidates: the best after the last, `top` times
  Key last = ~0ull;
  for (int r = 0; r < top; ++r) {
    Key k = 0;
    for (int i = threadIdx.x; i < keys; i += NJ)
      if (from[i] < last) k = max(k, from[i]);
    k = best_of_wave(k);
    __syncthreads();
    if (lane == 0) list[threadIdx.x / 64] = k;
    __syncthreads();
    for (int w = 0; w < NJ / 64; ++w) k = max(k, list[w]);
    if (threadIdx.x == 0) put(r, k);
    last = k;
  }
}

template <int TYPE>
void launch_type(const LogprobPlan& p, const void* logits, int64_t row_stride, int n, int vocab, const int32_t* tokens,
                 int top, float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace,
                 hipStream_t st) {
  typedef typename Elem<TYPE>::T T;
  ChunkStat* stats = (ChunkStat*)workspace;
  Key* best = (Key*)((char*)workspace + ((size_t)n * p.chunks * sizeof(ChunkStat) + 255) / 256 * 256);
  hipLaunchKernelGGL(logprob_chunk_kernel<TYPE>, dim3((unsigned)((int64_t)n * p.chunks)), dim3(NT), 0, st,
                     (const T*)logits, row_stride, vocab, p.chunks, top, stats, best);
  hipLaunchKernelGGL(logprob_join_kernel<TYPE>, dim3(n), dim3(NJ), 0, st, (const T*)logits, row_stride, vocab, p.chunks,
                     top, stats, best, tokens, logprob, entropy, top_ids, top_logprobs);
}

}  // namespace

LogprobPlan logprob_plan(int type, int n, int vocab, int top) {
  LogprobPlan p;
  const int skew = type == AMK_F32 ? 3 : 7;  // entries a row may begin after a 16-byte boundary
  p.chunks = (vocab + skew + NT * PER - 1) / (NT * PER);
  const size_t all = (size_t)n * p.chunks;
  p.workspace = (all * sizeof(ChunkStat) + 255) / 256 * 256 + all * top * sizeof(Key);
  return p;
}

int launch_logprobs(const LogprobPlan& p, const void* logits, int type, int64_t row_stride, int n, int vocab,
                    const int32_t* tokens, int top, float* logprob, float* entropy, int32_t* top_ids,
                    float* top_logprobs, void* workspace, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (type == AMK_F32)
    launch_type<AMK_F32>(p, logits, row_stride, n, vocab, tokens, top, logprob, entropy, top_ids, top_logprobs, workspace, st);
  else if (type == AMK_BF16)
    launch_type<AMK_BF16>(p, logits, row_stride, n, vocab, tokens, top, logprob, entropy, top_ids, top_logprobs, workspace, st);
  else
    launch_type<AMK_F16>(p, logits, row_stride, n, vocab, tokens, top, logprob, entropy, top_ids, top_logprobs, workspace, st);
  return hipGetLastError() == hipSuccess ? AMK_OK : AMK_ERR_DEVICE;
}

}  // namespace amk
