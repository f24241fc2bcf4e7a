// C ABI of the operators for several tokens: argument checks and launches.
#include <cmath>

#include "ops.h"

using namespace amk;

namespace {

constexpr int64_t kMostThreads = 0xffffffff;  // of a grid
constexpr int64_t kMostRows = 1 << 30;  // of an attention: kernels add to row numbers in 32 bits

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0; }

// Shapes and operands that both attentions share; keys == 0 leaves k and v unread.
int check_attention(const amk_attention_t* a, int64_t total_q, int64_t keys) {
  if (!a || !a->q || !a->out || (keys > 0 && (!a->k || !a->v))) return AMK_ERR_INVALID_ARGUMENT;
  if (a->n_heads < 1 || a->n_kv_heads < 1) return AMK_ERR_INVALID_ARGUMENT;
  if (a->n_heads % a->n_kv_heads || (a->head_dim != 64 && a->head_dim != 128)) return AMK_ERR_UNSUPPORTED;
  if (!(a->scale > 0.f) || !std::isfinite(a->scale)) return AMK_ERR_INVALID_ARGUMENT;
  for (const void* p : {a->q, a->k, a->v, (const void*)a->out})
    if (!aligned(p, 16)) return AMK_ERR_INVALID_ARGUMENT;
  for (int64_t s : {a->q_token, a->q_head, a->k_token, a->k_head, a->v_token, a->v_head, a->out_token, a->out_head})
    if (!stride_ok(s)) return AMK_ERR_INVALID_ARGUMENT;
  if (total_q * a->n_heads > kMostRows || keys > kMostRows || a->k_token > 1 << 24 || a->v_token > 1 << 24)
    return AMK_ERR_UNSUPPORTED;
  return AMK_OK;
}

bool shape_ok(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int64_t total_q, int64_t keys) {
  return n_heads > 0 && n_kv_heads > 0 && n_heads % n_kv_heads == 0 && (head_dim == 64 || head_dim == 128) &&
         total_q * n_heads <= kMostRows && keys <= kMostRows;
}

bool grid_ok(const AttnPlan& p, int32_t n_kv_heads) {
  return (int64_t)p.tiles * p.splits * n_kv_heads <= kMostThreads / (64 * p.waves);
}

int check_workspace(const void* p, size_t have, size_t need) {
  if (need == 0) return AMK_OK;
  return p && aligned(p, 256) && have >= need ? AMK_OK : AMK_ERR_INVALID_ARGUMENT;
}

}  // namespace

extern "C" {

int amk_linear(const void* x, int64_t x_stride, int32_t n, int32_t in, int32_t out, const void* w, const void* scale,
               int32_t weight_format, int32_t group_size, void* y, int64_t y_stride, int32_t y_type, int32_t accumulate,
               void* stream) {
  if (n < 0 || out < 0 || in < 1 || accumulate < 0 || accumulate > 1) return AMK_ERR_INVALID_ARGUMENT;
  if (weight_format < AMK_WEIGHTS_BF16 || weight_format > AMK_WEIGHTS_W4A16) return AMK_ERR_INVALID_ARGUMENT;
  if (y_type != AMK_F32 && y_type != AMK_BF16) return AMK_ERR_INVALID_ARGUMENT;
  const bool w4 = weight_format == AMK_WEIGHTS_W4A16;
  const int group = group_size ? group_size : 128;
  if (w4 && (group < 32 || group > 1024 || (group & (group - 1)))) return AMK_ERR_INVALID_ARGUMENT;
  if (in % 16 || (w4 && in % group) || in > 1 << 22 || x_stride > 1 << 22) return AMK_ERR_UNSUPPORTED;
  if (n == 0 || out == 0) return AMK_OK;
  if (!x || !w || !y || !aligned(x, 16) || !aligned(w, 16) || x_stride < in || x_stride % 8 || y_stride < out ||
      !aligned(y, y_type == AMK_F32 ? 4 : 2))
    return AMK_ERR_INVALID_ARGUMENT;
  if (weight_format != AMK_WEIGHTS_BF16 && (!scale || !aligned(scale, w4 ? 2 : 4))) return AMK_ERR_INVALID_ARGUMENT;
  if (out > 1 << 26 || ((int64_t)n + 127) / 128 * (((int64_t)out + 127) / 128) > kMostThreads / 512)
    return AMK_ERR_UNSUPPORTED;
  LinearArgs a = {};
  a.x = (const uint16_t*)x; a.x_stride = x_stride; a.n = n; a.in = in;
  a.part[0] = {w, scale, y, out}; a.parts = 1;
  a.fmt = weight_format; a.group = group; a.y_stride = y_stride; a.y_bf16 = y_type == AMK_BF16;
  a.accumulate = accumulate;
  return launch_linear(a, stream);
}

size_t amk_prompt_attention_workspace(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_seqs,
                                      int32_t total_q, int32_t total_k) {
  if (n_seqs < 1 || total_q < 1 || total_k < 0 || !shape_ok(n_heads, n_kv_heads, head_dim, total_q, total_k)) return 0;
  return prompt_plan(n_heads, n_kv_heads, head_dim, n_seqs, total_q, total_k).workspace;
}

int amk_prompt_attention(const amk_attention_t* a, const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs,
                         int32_t total_q, int32_t total_k, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a || total_q < 0 || total_k < 0 || n_seqs < 0) return AMK_ERR_INVALID_ARGUMENT;
  if (cu_q ? !cu_k || !aligned(cu_q, 4) || !aligned(cu_k, 4) : cu_k || n_seqs != 1) return AMK_ERR_INVALID_ARGUMENT;
  if (total_q == 0 || n_seqs == 0) return AMK_OK;
  int st = check_attention(a, total_q, total_k);
  if (st != AMK_OK) return st;
  const AttnPlan p = prompt_plan(a->n_heads, a->n_kv_heads, a->head_dim, n_seqs, total_q, total_k);
  if (!grid_ok(p, a->n_kv_heads)) return AMK_ERR_UNSUPPORTED;
  st = check_workspace(workspace, workspace_bytes, p.workspace);
  if (st != AMK_OK) return st;
  return launch_prompt(*a, p, cu_q, cu_k, n_seqs, total_q, total_k, workspace, stream);
}

size_t amk_tree_attention_workspace(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n, int32_t pos) {
  if (n < 1 || n > AMK_TREE_MAX || pos < 0 || !shape_ok(n_heads, n_kv_heads, head_dim, n, (int64_t)pos + n)) return 0;
  return tree_plan(n_heads, n_kv_heads, head_dim, n, pos).workspace;
}

int amk_tree_attention(const amk_attention_t* a, int32_t n, int32_t pos, const uint64_t* masks, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (!a || n < 0 || n > AMK_TREE_MAX || pos < 0 || pos > INT32_MAX - n) return AMK_ERR_INVALID_ARGUMENT;
  if (n == 0) return AMK_OK;
  if (!masks) return AMK_ERR_INVALID_ARGUMENT;
  int st = check_attention(a, n, (int64_t)pos + n);
  if (st != AMK_OK) return st;
  const AttnPlan p = tree_plan(a->n_heads, a->n_kv_heads, a->head_dim, n, pos);
  if (!grid_ok(p, a->n_kv_heads)) return AMK_ERR_UNSUPPORTED;
  st = check_workspace(workspace, workspace_bytes, p.workspace);
  if (st != AMK_OK) return st;
  TreeMasks m = {};
  for (int i = 0; i < n; ++i) m.bits[i] = n == 64 ? masks[i] : masks[i] & ((1ull << n) - 1);
  return launch_tree(*a, p, n, pos, m, workspace, stream);
}

size_t amk_token_logprobs_workspace(int32_t type, int32_t n, int32_t vocab, int32_t top) {
  if (type < AMK_F32 || type > AMK_F16 || n < 1 || vocab < 1 || vocab > 1 << 20 || top < 0 || top > AMK_TOP_MAX) return 0;
  return logprob_plan(type, n, vocab, top).workspace;
}

int amk_token_logprobs(const void* logits, int32_t type, int64_t row_stride, int32_t n, int32_t vocab,
                       const int32_t* tokens, int32_t top, float* logprob, float* entropy, int32_t* top_ids,
                       float* top_logprobs, void* workspace, size_t workspace_bytes, void* stream) {
  if (type < AMK_F32 || type > AMK_F16 || n < 0 || vocab < 1 || vocab > 1 << 20 || top < 0 || top > AMK_TOP_MAX ||
      top > vocab)
    return AMK_ERR_INVALID_ARGUMENT;
  if (n == 0) return AMK_OK;
  if (!logits || !aligned(logits, type == AMK_F32 ? 4 : 2) || (n > 1 && row_stride < vocab)) return AMK_ERR_INVALID_ARGUMENT;
  if ((tokens != nullptr) != (logprob != nullptr) || (top && (!top_ids || !top_logprobs))) return AMK_ERR_INVALID_ARGUMENT;
  for (const void* p : {(const void*)tokens, (const void*)logprob, (const void*)entropy, (const void*)top_ids,
                        (const void*)top_logprobs})
    if (!aligned(p, 4)) return AMK_ERR_INVALID_ARGUMENT;
  const LogprobPlan p = logprob_plan(type, n, vocab, top);
  if ((int64_t)n * p.chunks > kMostThreads / 256) return AMK_ERR_UNSUPPORTED;
  const int st = check_workspace(workspace, workspace_bytes, p.workspace);
  if (st != AMK_OK) return st;
  return launch_logprobs(p, logits, type, row_stride, n, vocab, tokens, top, logprob, entropy, top_ids, top_logprobs,
                         workspace, stream);
}

int amk_kv_keep(void* kv_cache, int32_t n_layers, int32_t n_kv_heads, int32_t max_seq, int32_t head_dim, int32_t pos,
                const int32_t* rows, int32_t count, void* stream) {
  if (n_layers < 1 || n_kv_heads < 1 || max_seq < 1 || pos < 0 || count < 0 || count > AMK_TREE_MAX)
    return AMK_ERR_INVALID_ARGUMENT;
  if (head_dim != 64 && head_dim != 128) return AMK_ERR_UNSUPPORTED;
  if (count == 0) return AMK_OK;
  if (!kv_cache || !rows || !aligned(kv_cache, 16)) return AMK_ERR_INVALID_ARGUMENT;
  if ((int64_t)n_layers * 2 * n_kv_heads > kMostThreads / 256) return AMK_ERR_UNSUPPORTED;
  TreeDepths r = {};
  for (int i = 0; i < count; ++i) {
    if (rows[i] < 0 || (i && rows[i] <= rows[i - 1]) || (int64_t)pos + rows[i] >= max_seq) return AMK_ERR_INVALID_ARGUMENT;
    r.at[i] = rows[i];
  }
  return launch_keep(kv_cache, n_layers * 2 * n_kv_heads, max_seq, head_dim, pos, r, count, stream);
}

}  // extern "C"
