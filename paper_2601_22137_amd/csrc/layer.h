// Declarations shared by the operators of a transformer layer (dropout, norm and rotation of queries and keys, attention) and of the ends
// of a model around them (embedding, norm of the residual stream, log-probabilities and losses).
#pragma once
#include "common.h"

namespace prism {

// Device memory of `bytes` bytes: the caller's, if it passed one, else the cached one of (device, stream).  PRISM_OK or an error.
int layer_workspace(size_t bytes, void* given, size_t given_bytes, hipStream_t s, char** out);
void set_last_error(const char* msg);

int launch_dropout(const void* x, const void* residual, void* y, long long n, int dt, unsigned limit, uint64_t seed, uint32_t offset, hipStream_t s);

// workgroups of prism_qk_norm_rope_backward, each with partial sums of the weights' gradients: eight per CU
constexpr int NR_MAX_BLOCKS = 2048;
int launch_norm_rope(const void* q, const void* k, void* qo, void* ko, int dt, const prism_norm_rope_desc& d, hipStream_t s);
size_t norm_rope_backward_bytes(const prism_norm_rope_desc& d);
int launch_norm_rope_backward(const void* dqo, const void* dko, const void* q, const void* k, void* dq, void* dk, float* dqw, float* dkw, int dt,
                              const prism_norm_rope_desc& d, float* part, hipStream_t s);

struct AttnPlan {
  int split;                            // parts of the keys of a row tile
  bool few;                             // at most 32 rows a pair: the kernel for single tokens
  int chunk, parts, items;              // rows of a part of a key tile's rows (0: whole), the most parts of a key tile, parts of a pair
  size_t o_part, o_ml, o_stat, total;   // bytes from the start of the workspace, where the ranges of the documents lie
};
AttnPlan attention_plan(const prism_attention_desc& d, int dt, bool backward);
void launch_doc_ranges(const prism_attention_desc& d, int4* to, hipStream_t s);
int launch_attention(const void* q, const void* k, const void* v, void* out, float* lse, int dt, const prism_attention_desc& d, char* ws, hipStream_t s);
int launch_attention_backward(const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, void* dq, void* dk,
                              void* dv, int dt, const prism_attention_desc& d, char* ws, hipStream_t s);

int launch_embedding(const void* table, const void* tokens, void* out, int dt, const prism_embedding_desc& d, hipStream_t s);
struct EmbeddingPlan {
  int chunks, tile, tiles;              // 64 vectors of 16 bytes each in a row; sorted tokens of a tile; tiles
  size_t o_sorted, o_part, total;       // bytes from the start of the workspace, where the starts of the rows' tokens lie
};
EmbeddingPlan embedding_plan(const prism_embedding_desc& d, int dt);
int launch_embedding_backward(const void* dout, const void* tokens, void* dtable, int dt, const prism_embedding_desc& d, char* ws, hipStream_t s);

int launch_layer_norm(const void* x, const void* residual, const float* weight, const float* bias, void* y, void* total, float* stats, int dt,
                      const prism_layer_norm_desc& d, hipStream_t s);
size_t layer_norm_backward_bytes(const prism_layer_norm_desc& d, int dt);
// part: partial sums of the gradients of weight and bias, or null where neither is wanted
int launch_layer_norm_backward(const void* dy, const void* total, const float* stats, const float* weight, const void* dtotal, void* dx, float* dweight,
                               float* dbias, int dt, const prism_layer_norm_desc& d, float* part, hipStream_t s);

int launch_logprob(const void* z, const void* tokens, float* logp, float* lse, int dt, const prism_logits_desc& d, hipStream_t s);
int launch_logprob_backward(const float* dlogp, const void* z, const void* tokens, const float* lse, void* dz, int dt, const prism_logits_desc& d, hipStream_t s);
size_t policy_loss_bytes(const prism_logits_desc& d);
int launch_policy_loss(const void* z, const void* tokens, float* loss, float* logp, float* lse, float* dlogp, void* dz, int dt, const prism_logits_desc& d, char* ws,
                       hipStream_t s);

}  // namespace prism
