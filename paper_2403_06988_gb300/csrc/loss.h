// loss.h -- the losses over the vocabulary and the embedding as the C ABI
// (host.cpp) launches them: loss.cu, distill.cu, embed.cu.
#pragma once
#include "domino_internal.h"

namespace domino {

// Rows of tokens, and tokens of a list: the kernels count them in 32 bits, in steps of a tile, a chunk (2^19 at most) or a
// CTA's threads beyond the last.
constexpr int32_t kMaxRows = INT32_MAX - (1 << 20);

// Cross entropy under the masked softmax of hidden . weight^T.
struct LossArgs {
    const void* hidden;        // bf16 [rows][hidden_stride]
    const void* weight;        // bf16 [n_tokens][weight_stride]
    int64_t hidden_stride, weight_stride;
    int32_t rows, dim, n_tokens;
    const uint32_t* mask;      // nullptr: every token allowed
    const int32_t* targets;
    float* loss;               // forward
    float* lse;                // forward: may be nullptr; gradient: given
    const float* grad_loss;    // gradient
    void* dhidden;
    void* dweight;
    int64_t dhidden_stride, dweight_stride;
    uint32_t* err;
};
// rows, dim and n_tokens at least 1, at most kMaxRows rows; tma_ready() operands need no copy.
bool loss_fits(const LossArgs& a);
size_t loss_workspace(const LossArgs& a, const LaunchEnv& env, bool grad);
cudaError_t launch_token_loss(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st);
cudaError_t launch_token_loss_grad(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st);
// Few rows (loss_few.cu): whether these are.
bool few_rows(const LossArgs& a);
size_t few_workspace(const LossArgs& a, const LaunchEnv& env, bool grad);
cudaError_t launch_few_loss(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st);
cudaError_t launch_few_loss_grad(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st);
// Rows' partials (max, sum of exp against it), `parts` each, into loss and lse.
cudaError_t launch_loss_merge(const LossArgs& a, const float2* part, int32_t parts, const float* target_logit,
                              cudaStream_t st);

// Divergence of a teacher's top logits from the masked softmax of a row.
struct DistillArgs {
    const void* logits;        // [rows][stride]
    int dtype;
    int64_t stride;
    int32_t rows, n_tokens;
    const uint32_t* mask;      // nullptr: every token allowed
    const void* teacher;       // [rows][k]
    int teacher_dtype;
    const int32_t* ids;        // [rows][k], below 0: no entry
    int32_t k;
    float temperature;
    float* loss;               // forward
    float* lse;                // forward: may be nullptr; gradient: given
    const float* grad_loss;    // gradient
    void* dlogits;             // gradient, the logits' type; may be `logits`
    int64_t dstride;
    uint32_t* err;
};
constexpr int kDistillMaxK = 1024;
cudaError_t launch_distill(const DistillArgs& a, const LaunchEnv& env, bool grad, cudaStream_t st);

// Rows of an embedding table.
struct EmbedArgs {
    const int32_t* tokens;
    int32_t n, n_tokens, dim;
    int dtype;
    float scale;
    const void* weight;        // [n_tokens][weight_stride]
    int64_t weight_stride;
    void* out;                 // [n][out_stride]
    int64_t out_stride;
    // gradient
    const void* grad;          // [n][grad_stride]
    int64_t grad_stride;
    void* dweight;             // [n_tokens][dweight_stride]
    int64_t dweight_stride;
    bool add;                  // to what dweight holds
    uint32_t* err;
};
cudaError_t launch_embed(const EmbedArgs& a, const LaunchEnv& env, cudaStream_t st);
size_t embed_workspace(const EmbedArgs& a, const LaunchEnv& env);
cudaError_t launch_embed_grad(const EmbedArgs& a, const LaunchEnv& env, void* space, cudaStream_t st);

}  // namespace domino
