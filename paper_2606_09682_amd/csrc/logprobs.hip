// Log probabilities of given tokens, entropy and the most probable alternatives
// of rows of logits.
//
// With m the row's maximum, s = sum e^(x - m) and u = sum (x - m) e^(x - m):
// log p(x) = x - m - log s and H = log s - u / s.  A workgroup takes a chunk of a
// row into registers in one read and leaves (m, s, u) and the chunk's best
// entries; a second kernel, one workgroup a row, joins the chunks.  One read of
// the logits is all that cannot be avoided, so HBM bounds large calls and the
// two launches small ones.
//
// Best entries.  Each lane's maximum over the workgroup's waves gives 64 maxima
// of disjoint groups; the top-th largest of them is a value that at least `top`
// entries reach, and few more do unless many are equal.  The entries that reach
// it are listed and ranked by counting.  Where they overflow the list (rows of
// few distinct values), `top` rounds each find the best entry after the last.
// Entries compare by value and then the lower index, so the result is one and
// the same however the list was filled.
#include <cmath>

#include "ops.h"
#include "ops_device.h"

namespace amk {
namespace {

constexpr int NT = 512, WAVES = NT / 64;
constexpr int LIST = 1024;  // entries ranked by counting

struct Best {
  float x;
  int32_t i;  // -1: none
};

// Whether a comes before b: the larger value, the lower index.
__device__ __forceinline__ bool before(const Best& a, const Best& b) {
  return a.i >= 0 && (b.i < 0 || a.x > b.x || (a.x == b.x && a.i < b.i));
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

// The workgroup's maximum (NaN left out) and sum; every thread gets them.
__device__ float block_max(float v, float* tmp) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  v = tmp[0];
  for (int i = 1; i < WAVES; ++i) v = fmaxf(v, tmp[i]);
  return v;
}
__device__ float block_sum(float v, float* tmp) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  v = tmp[0];
  for (int i = 1; i < WAVES; ++i) v += tmp[i];
  return v;
}

// Ranks `count` listed entries and writes the best `top` in order (none: i = -1).
__device__ void rank_list(const Best* list, int count, int top, Best* out) {
  for (int c = threadIdx.x; c < count; c += NT) {
    const Best b = list[c];
    int rank = 0;
    for (int o = 0; o < count; ++o) rank += before(list[o], b);
    if (b.i >= 0 && rank < top) out[rank] = b;
  }
}

// The statistics of one chunk, then its best entries.
struct ChunkStat {
  float m, s, u;
  int32_t nan;
};

template <int TYPE, int PER>
__global__ void __launch_bounds__(NT) logprob_chunk_kernel(const typename Elem<TYPE>::T* logits, int64_t row_stride,
                                                           int vocab, int chunks, int top, ChunkStat* stats,
                                                           Best* best) {
  typedef typename Elem<TYPE>::T T;
  constexpr int VEC = 16 / sizeof(T);
  __shared__ float tmp[WAVES];
  __shared__ float lane_max[WAVES][64];
  __shared__ Best list[LIST];
  __shared__ Best out[AMK_TOP_MAX];
  __shared__ int count;
  __shared__ float reach;
  __shared__ Best found[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const T* p = logits + (int64_t)row * row_stride;
  // chunks are cut at 16-byte boundaries of memory: `skew` entries before the row
  const int skew = (int)(((uintptr_t)p & 15) / sizeof(T));
  const int first = chunk * (NT * PER) - skew;

  float x[PER];
  int at0[PER / VEC];
#pragma unroll
  for (int j = 0; j < PER / VEC; ++j) {
    const int i = first + (j * NT + (int)threadIdx.x) * VEC;
    at0[j] = i;
    if (i >= 0 && i + VEC <= vocab) {
      const u32x4 v = *(const u32x4*)(p + i);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const uint32_t word = v[sizeof(T) == 4 ? e % 4 : e / 2 % 4];
        x[j * VEC + e] = Elem<TYPE>::bits(sizeof(T) == 4 ? word : word >> (e % 2 * 16));
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        x[j * VEC + e] = i + e >= 0 && i + e < vocab ? Elem<TYPE>::get(p[i + e]) : -INFINITY;
    }
  }

  float mine = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    mine = fmaxf(mine, x[j]);
    nan |= x[j] != x[j];
  }
  const float m = block_max(mine, tmp);
  float s = 0.f, u = 0.f;
  if (m > -INFINITY) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const float z = x[j] - m, e = __expf(z);
      s += e;
      u += e > 0.f ? z * e : 0.f;
    }
  }
  s = block_sum(s, tmp);
  u = block_sum(u, tmp);
  nan = __syncthreads_or(nan);
  if (threadIdx.x == 0) stats[blockIdx.x] = {m, s, u, nan};
  if (top == 0 || nan) return;

  lane_max[wave][lane] = mine;
  if (threadIdx.x < AMK_TOP_MAX) out[threadIdx.x] = {-INFINITY, -1};
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  if (wave == 0) {
    float g = lane_max[0][lane];
    for (int i = 1; i < WAVES; ++i) g = fmaxf(g, lane_max[i][lane]);
    int rank = 0;
    for (int o = 0; o < 64; ++o) {
      const float v = __shfl(g, o);
      rank += v > g || (v == g && o < lane);
    }
    if (rank == top - 1) reach = g;
  }
  __syncthreads();
  const float least = reach;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = at0[j / VEC] + j % VEC;
    if (x[j] >= least && i >= 0 && i < vocab) {
      const int c = atomicAdd(&count, 1);
      if (c < LIST) list[c] = {x[j], i};
    }
  }
  __syncthreads();
  if (count <= LIST) {
    rank_list(list, count, top, out);
  } else {
    Best last = {INFINITY, -1};
    for (int r = 0; r < top; ++r) {
      Best b = {-INFINITY, -1};
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const Best c = {x[j], at0[j / VEC] + j % VEC};
        if (c.i >= 0 && c.i < vocab && (r == 0 || before(last, c)) && before(c, b)) b = c;
      }
      for (int d = 32; d; d >>= 1) {
        const Best c = {__shfl_xor(b.x, d), __shfl_xor(b.i, d)};
        if (before(c, b)) b = c;
      }
      if (lane == 0) found[wave] = b;
      __syncthreads();
      b = found[0];
      for (int i = 1; i < WAVES; ++i)
        if (before(found[i], b)) b = found[i];
      if (threadIdx.x == 0) out[r] = b;
      last = b;
      __syncthreads();
      if (b.i < 0) break;
    }
  }
  __syncthreads();
  if (threadIdx.x < top) best[(int64_t)blockIdx.x * top + threadIdx.x] = out[threadIdx.x];
}

template <int TYPE>
__global__ void __launch_bounds__(NT) logprob_join_kernel(const typename Elem<TYPE>::T* logits, int64_t row_stride,
                                                          int vocab, int chunks, int top, const ChunkStat* stats,
                                                          const Best* best, const int32_t* tokens, float* logprob,
                                                          float* entropy, int32_t* top_ids, float* top_logprobs) {
  __shared__ float tmp[WAVES];
  __shared__ Best list[LIST];
  __shared__ Best out[AMK_TOP_MAX];
  const int row = blockIdx.x;
  const ChunkStat* st = stats + (int64_t)row * chunks;
  float m = -INFINITY;
  bool nan = false;
  for (int c = threadIdx.x; c < chunks; c += NT) {
    m = fmaxf(m, st[c].m);
    nan |= st[c].nan != 0;
  }
  m = block_max(m, tmp);
  nan = __syncthreads_or(nan) || m == INFINITY || m == -INFINITY;
  float s = 0.f, u = 0.f;
  for (int c = threadIdx.x; c < chunks; c += NT) {
    // a chunk's sums move to the row's maximum: x - m = (x - mc) + (mc - m)
    if (st[c].m == -INFINITY) continue;
    const float d = st[c].m - m, f = __expf(d);
    s += st[c].s * f;
    u += f > 0.f ? (st[c].u + d * st[c].s) * f : 0.f;
  }
  s = block_sum(s, tmp);
  u = block_sum(u, tmp);
  const float ls = logf(s), none = __builtin_nanf("");
  if (threadIdx.x == 0) {
    if (entropy) entropy[row] = nan ? none : ls - u / s;
    if (tokens) {
      const int t = tokens[row];
      float lp = none;
      if (!nan && t >= 0 && t < vocab) lp = Elem<TYPE>::get(logits[row * row_stride + t]) - m - ls;
      logprob[row] = lp;
    }
  }
  if (top == 0) return;
  if (threadIdx.x < AMK_TOP_MAX) out[threadIdx.x] = {none, -1};
  int count = 0;
  if (!nan) {
    // list the chunks' entries, as many chunks at a time as the list holds beside the best so far
    const int per = (LIST - AMK_TOP_MAX) / top;
    for (int c0 = 0; c0 < chunks; c0 += per) {
      const int n = min(per, chunks - c0) * top;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += NT) list[count + i] = best[((int64_t)row * chunks + c0) * top + i];
      __syncthreads();
      rank_list(list, count + n, top, out);
      __syncthreads();
      if (threadIdx.x < top) list[threadIdx.x] = out[threadIdx.x];
      count = top;
    }
  }
  __syncthreads();
  if (threadIdx.x < top) {
    const Best b = out[threadIdx.x];
    top_ids[(int64_t)row * top + threadIdx.x] = b.i;
    top_logprobs[(int64_t)row * top + threadIdx.x] = b.i < 0 ? none : b.x - m - ls;
  }
}

template <int TYPE>
void launch_type(const LogprobPlan& p, const void* logits, int64_t row_stride, int n, int vocab, const int32_t* tokens,
                 int top, float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace,
                 hipStream_t st) {
  typedef typename Elem<TYPE>::T T;
  ChunkStat* stats = (ChunkStat*)workspace;
  Best* best = (Best*)((char*)workspace + ((size_t)n * p.chunks * sizeof(ChunkStat) + 255) / 256 * 256);
  const dim3 grid((unsigned)((int64_t)n * p.chunks));
  if (p.chunk == NT * 32)
    hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 32>), grid, dim3(NT), 0, st, (const T*)logits, row_stride, vocab,
                       p.chunks, top, stats, best);
  else
    hipLaunchKernelGGL((logprob_chunk_kernel<TYPE, 8>), grid, dim3(NT), 0, st, (const T*)logits, row_stride, vocab,
                       p.chunks, top, stats, best);
  hipLaunchKernelGGL(logprob_join_kernel<TYPE>, dim3(n), dim3(NT), 0, st, (const T*)logits, row_stride, vocab, p.chunks,
                     top, stats, best, tokens, logprob, entropy, top_ids, top_logprobs);
}

}  // namespace

LogprobPlan logprob_plan(int type, int n, int vocab, int top) {
  LogprobPlan p;
  const int skew = type == AMK_F32 ? 3 : 7;  // entries a row may begin after a 16-byte boundary
  // large chunks where they fill the GPU, small ones for few rows
  p.chunk = NT * 32;
  p.chunks = (vocab + skew + p.chunk - 1) / p.chunk;
  if ((int64_t)n * p.chunks < 512) {
    p.chunk = NT * 8;
    p.chunks = (vocab + skew + p.chunk - 1) / p.chunk;
  }
  const size_t all = (size_t)n * p.chunks;
  p.workspace = (all * sizeof(ChunkStat) + 255) / 256 * 256 + all * top * sizeof(Best);
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
