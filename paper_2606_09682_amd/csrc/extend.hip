// Elementwise kernels of amk_extend, and the rows of a KV cache moved together.
// All of them read and write each byte once (the norm reads its row twice, the
// second time from L2) and are bound by HBM at thousands of tokens and by their launch at
// few: keeping 7 rows in 512 planes of 128-wide heads takes 2.8 us for 1.8 MB.
#include "ops.h"
#include "ops_device.h"

namespace amk {
namespace {

// x[t] = the embedding row of token t, widened to fp32
__global__ void __launch_bounds__(256) embed_kernel(const uint16_t* embed, const TokenBlock t, int hidden, float* x) {
  const uint16_t* row = embed + (int64_t)t.id[blockIdx.x] * hidden;
  float* to = x + (int64_t)blockIdx.x * hidden;
  for (int i = threadIdx.x * 4; i < hidden; i += 1024) {  // hidden is a multiple of 16
    const u32x2 v = *(const u32x2*)(row + i);
    const f32x4 f = {bf16_to_f32((uint16_t)v[0]), bf16_to_f32((uint16_t)(v[0] >> 16)), bf16_to_f32((uint16_t)v[1]),
                     bf16_to_f32((uint16_t)(v[1] >> 16))};
    *(f32x4*)(to + i) = f;
  }
}

// h[t] = x[t] / sqrt(mean(x[t]^2) + eps) * gain in fp32, rounded to bf16 for the products
__global__ void __launch_bounds__(256) rmsnorm_kernel(const float* x, const uint16_t* gain, int hidden, float eps,
                                                      uint16_t* h) {
  __shared__ float tmp[4];
  const float* row = x + (int64_t)blockIdx.x * hidden;
  float s = 0.f;
  for (int i = threadIdx.x * 4; i < hidden; i += 1024) {
    const f32x4 v = *(const f32x4*)(row + i);
    s += v[0] * v[0] + v[1] * v[1] + v[2] * v[2] + v[3] * v[3];
  }
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = s;
  __syncthreads();
  const float r = 1.f / sqrtf((tmp[0] + tmp[1] + tmp[2] + tmp[3]) / (float)hidden + eps);
  uint16_t* to = h + (int64_t)blockIdx.x * hidden;
  for (int i = threadIdx.x * 4; i < hidden; i += 1024) {
    const f32x4 v = *(const f32x4*)(row + i);
    const u32x2 g = *(const u32x2*)(gain + i);
    const u32x2 o = {pack_bf16(v[0] * r * bf16_to_f32((uint16_t)g[0]), v[1] * r * bf16_to_f32((uint16_t)(g[0] >> 16))),
                     pack_bf16(v[2] * r * bf16_to_f32((uint16_t)g[1]), v[3] * r * bf16_to_f32((uint16_t)(g[1] >> 16)))};
    *(u32x2*)(to + i) = o;
  }
}

// One token's projections [q heads][k heads][v heads][hd]: q and k turned by RoPE
// (pairs i, i + hd / 2) to the token's position, q rounded to bf16 for the
// attention, k and v rounded and appended to the layer's cache.
template <bool TREE>
__global__ void __launch_bounds__(256) rope_append_kernel(const float* qkv, const float2* rope, int pos,
                                                          const TreeDepths depths, int nq, int nkv, int half,
                                                          int max_seq, uint16_t* q, uint16_t* k, uint16_t* v) {
  const int t = blockIdx.x, slots = nq + 2 * nkv, hd = 2 * half;
  const float2* turn = rope + (int64_t)(pos + (TREE ? depths.at[t] : t)) * half;
  for (int u = threadIdx.x; u < slots * half; u += 256) {
    const int s = u / half, i = u % half;
    const float* from = qkv + ((int64_t)t * slots + s) * hd;
    float a = from[i], b = from[i + half];
    if (s < nq + nkv) {
      const float2 cs = turn[i];
      const float x = a * cs.x - b * cs.y, y = b * cs.x + a * cs.y;
      a = x;
      b = y;
    }
    uint16_t* to;
    if (s < nq) to = q + ((int64_t)t * nq + s) * hd;
    else if (s < nq + nkv) to = k + ((int64_t)(s - nq) * max_seq + pos + t) * hd;
    else to = v + ((int64_t)(s - nq - nkv) * max_seq + pos + t) * hd;
    to[i] = f32_to_bf16(a);
    to[i + half] = f32_to_bf16(b);
  }
}

// a = silu(gate) * up, rounded to bf16 for the product
__global__ void __launch_bounds__(256) silu_mul_kernel(const float* gate, const float* up, int64_t count, uint16_t* a) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= count) return;  // count is a multiple of 16
  const f32x4 g = *(const f32x4*)(gate + i), u = *(const f32x4*)(up + i);
  float r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = g[e] / (1.f + __expf(-g[e])) * u[e];
  const u32x2 o = {pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
  *(u32x2*)(a + i) = o;
}

// One workgroup per plane (layer, K or V, head): every row is in LDS before the
// first is written, so rows may move onto each other.
__global__ void __launch_bounds__(256) keep_kernel(uint16_t* kv, int64_t plane, int head_dim, int pos,
                                                   const TreeDepths rows, int count) {
  __shared__ u32x4 held[AMK_TREE_MAX * 128 / 8];
  uint16_t* base = kv + blockIdx.x * plane + (int64_t)pos * head_dim;
  const int per = head_dim / 8;
  for (int c = threadIdx.x; c < count * per; c += 256)
    held[c] = *(const u32x4*)(base + (int64_t)rows.at[c / per] * head_dim + c % per * 8);
  __syncthreads();
  for (int c = threadIdx.x; c < count * per; c += 256) *(u32x4*)(base + c * 8) = held[c];
}

int launched() { return hipGetLastError() == hipSuccess ? AMK_OK : AMK_ERR_DEVICE; }

}  // namespace

int launch_embed(const uint16_t* embed, const TokenBlock& t, int n, int hidden, float* x, void* stream) {
  hipLaunchKernelGGL(embed_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, embed, t, hidden, x);
  return launched();
}

int launch_rmsnorm(const float* x, const uint16_t* gain, int n, int hidden, float eps, uint16_t* h, void* stream) {
  hipLaunchKernelGGL(rmsnorm_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, x, gain, hidden, eps, h);
  return launched();
}

int launch_rope_append(const float* qkv, const float2* rope, int n, int pos, const TreeDepths* depths, int n_heads,
                       int n_kv_heads, int head_dim, int max_seq, uint16_t* q, uint16_t* k, uint16_t* v, void* stream) {
  const TreeDepths none = {};
  if (depths)
    hipLaunchKernelGGL(rope_append_kernel<true>, dim3(n), dim3(256), 0, (hipStream_t)stream, qkv, rope, pos, *depths,
                       n_heads, n_kv_heads, head_dim / 2, max_seq, q, k, v);
  else
    hipLaunchKernelGGL(rope_append_kernel<false>, dim3(n), dim3(256), 0, (hipStream_t)stream, qkv, rope, pos, none,
                       n_heads, n_kv_heads, head_dim / 2, max_seq, q, k, v);
  return launched();
}

int launch_silu_mul(const float* gate, const float* up, int64_t count, uint16_t* a, void* stream) {
  hipLaunchKernelGGL(silu_mul_kernel, dim3((unsigned)((count + 1023) / 1024)), dim3(256), 0, (hipStream_t)stream, gate,
                     up, count, a);
  return launched();
}

int launch_keep(void* kv, int planes, int max_seq, int head_dim, int pos, const TreeDepths& rows, int count,
                void* stream) {
  hipLaunchKernelGGL(keep_kernel, dim3(planes), dim3(256), 0, (hipStream_t)stream, (uint16_t*)kv,
                     (int64_t)max_seq * head_dim, head_dim, pos, rows, count);
  return launched();
}

}  // namespace amk
