// norm.h -- the root-mean-square norm, 8-bit codes and the logits of 8-bit operands as
// the C ABI (host.cpp) launches them: norm.cu, quantize8.cu, logits8.cu; and the decode
// under penalties (penalized.cu).
#pragma once
#include "domino_internal.h"

namespace domino {

// Rows of a stream.
struct NormArgs {
    const void* x;             // [rows][x_stride]
    const void* residual;      // [rows][residual_stride]; nullptr: none
    const void* weight;        // [dim]
    void* sum;                 // x + residual, rounded; nullptr without a residual
    int64_t x_stride, residual_stride, sum_stride;
    int32_t rows, dim;
    int dtype;
    float eps;
    // in the stream's type
    void* y;
    int64_t y_stride;
    float* rstd;               // [rows], may be nullptr
    // in codes
    uint8_t* codes;            // rows on 16-byte boundaries; nullptr: y
    int64_t codes_stride;
    float* scales;             // [rows][ceil(dim / 128)]
};
cudaError_t launch_norm(const NormArgs& a, const LaunchEnv& env, cudaStream_t st);

struct NormGradArgs {
    const void* h;             // the norm's input: x + residual
    const void* weight;
    const float* rstd;
    const void* dy;
    const void* dsum;          // nullptr: none
    void* dx;
    void* dweight;             // [dim]
    int64_t h_stride, dy_stride, dsum_stride, dx_stride;
    int32_t rows, dim;
    int dtype;
};
size_t norm_grad_workspace(const NormGradArgs& a, const LaunchEnv& env);
cudaError_t launch_norm_grad(const NormGradArgs& a, const LaunchEnv& env, void* space, cudaStream_t st);

struct Quantize8Args {
    const void* x;
    int64_t stride;
    int32_t rows, dim;
    int dtype;
    int32_t block;             // rows that share a scale: 1 or 128
    uint8_t* codes;            // rows on 16-byte boundaries
    int64_t codes_stride;
    float* scales;             // [ceil(rows / block)][ceil(dim / 128)]
};
cudaError_t launch_quantize8(const Quantize8Args& a, const LaunchEnv& env, cudaStream_t st);

struct Logits8Args {
    const uint8_t* hidden;     // [rows][hidden_stride], on 16-byte boundaries
    const uint8_t* weight;     // [n_tokens][weight_stride], on 16-byte boundaries
    const float* hidden_scales;
    const float* weight_scales;
    int64_t hidden_stride, weight_stride;
    int32_t rows, dim, n_tokens;
    int dtype;                 // of the logits
    void* logits;
    int64_t logits_stride;
    uint32_t* err;
};
bool logits8_fits(const Logits8Args& a);
cudaError_t launch_logits8(const Logits8Args& a, const LaunchEnv& env, cudaStream_t st);

constexpr int kMaxBias = 1024;
struct PenalizedArgs {
    const void* logits;
    int64_t stride;
    int32_t batch, n_tokens;
    int dtype;
    domino_penalties p;
    const uint32_t* mask;      // nullptr: every token allowed
    int32_t* argmax;
    float* lse;
    float* logprobs;
    const SampleArgs* sample;  // nullptr: greedy
    uint32_t* err;
};
cudaError_t launch_penalized(const PenalizedArgs& a, const LaunchEnv& env, cudaStream_t st);

}  // namespace domino
