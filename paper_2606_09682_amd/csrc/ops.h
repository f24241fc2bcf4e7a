// Internal launch interface of the operators for several tokens: arguments are
// already checked (ops_api.cpp) when these are called.
#pragma once

#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "../../include/amk.h"

namespace amk {

// One of the matrices a launch multiplies the same x with.
struct LinearPart {
  const void* w;
  const void* scale;
  void* y;
  int32_t out;
};

struct LinearArgs {
  const uint16_t* x;
  int64_t x_stride;
  int32_t n, in;
  LinearPart part[3];
  int32_t parts;      // of them used
  int32_t fmt;
  int32_t group;      // W4A16: columns per scale
  int64_t y_stride;   // of every y
  int32_t y_bf16, accumulate;
};

// How an attention is cut: row tiles of 32 * waves rows (a row is a query of one
// token and one head of a KV group), the keys of each tile in `splits` ranges.
struct AttnPlan {
  int32_t waves;
  int32_t tiles;      // row tiles per KV head (an upper bound for packed sequences)
  int32_t splits;
  size_t workspace;   // partial results, 0 for one split
};

AttnPlan prompt_plan(int n_heads, int n_kv_heads, int head_dim, int n_seqs, int total_q, int total_k);
AttnPlan tree_plan(int n_heads, int n_kv_heads, int head_dim, int n, int pos);
// No plan of these heads needs more workspace.
size_t attention_workspace_most(int n_heads, int n_kv_heads, int head_dim);

struct TreeMasks {
  uint64_t bits[AMK_TREE_MAX];
};

// Tree depths of up to AMK_TREE_MAX tokens, passed by value to kernels.
struct TreeDepths {
  int32_t at[AMK_TREE_MAX];
};

constexpr int kTokensPerLaunch = 512;  // 2 KiB of kernel arguments
struct TokenBlock {
  int32_t id[kTokensPerLaunch];
};

struct LogprobPlan {
  int32_t chunks;     // workgroups per row
  size_t workspace;
};

LogprobPlan logprob_plan(int type, int n, int vocab, int top);

int launch_linear(const LinearArgs& a, void* stream);
int launch_prompt(const amk_attention_t& a, const AttnPlan& p, const int32_t* cu_q, const int32_t* cu_k, int n_seqs,
                  int total_q, int total_k, void* workspace, void* stream);
int launch_tree(const amk_attention_t& a, const AttnPlan& p, int n, int pos, const TreeMasks& m, void* workspace,
                void* stream);
int launch_logprobs(const LogprobPlan& p, const void* logits, int type, int64_t row_stride, int n, int vocab,
                    const int32_t* tokens, int top, float* logprob, float* entropy, int32_t* top_ids,
                    float* top_logprobs, void* workspace, void* stream);
int launch_keep(void* kv, int planes, int max_seq, int head_dim, int pos, const TreeDepths& rows, int count,
                void* stream);

// Elementwise kernels of amk_extend.
int launch_embed(const uint16_t* embed, const TokenBlock& t, int n, int hidden, float* x, void* stream);
int launch_rmsnorm(const float* x, const uint16_t* gain, int n, int hidden, float eps, uint16_t* h, void* stream);
int launch_rope_append(const float* qkv, const float2* rope, int n, int pos, const TreeDepths* depths, int n_heads,
                       int n_kv_heads, int head_dim, int max_seq, uint16_t* q, uint16_t* k, uint16_t* v, void* stream);
int launch_silu_mul(const float* gate, const float* up, int64_t count, uint16_t* a, void* stream);

}  // namespace amk
