// From a model's tokens to its loss: embeddings, linear layers on 8-bit codes, the loss over the vocabulary.
#pragma once
#include "block.hpp"
#include "token_plan.hpp"

namespace onecomp {
namespace token {

using block::Rows;

onecomp_status quantize_tokens_run(onecomp_dtype dtype, const Rows& x, int64_t tokens, int64_t width, int8_t* codes, float* scales, int32_t* sums,
                                   hipStream_t stream);

struct Linear {
    const int8_t* codes;
    const float* token_scales;
    const int32_t* token_sums;
    const uint8_t* q;
    const float *scales, *zeros;
    const void* bias;
    Rows y;
    int64_t tokens, d_out, d_in;
};
onecomp_status linear_run(onecomp_dtype dtype, const Linear& P, hipStream_t stream);

onecomp_status embedding_forward_run(onecomp_dtype dtype, const int32_t* tokens, int64_t n, const Rows& table, int64_t vocab, int64_t width, float scale,
                                     const Rows& out, hipStream_t stream);
size_t embedding_workspace_bytes(int64_t n, int64_t vocab, int64_t width);
// base: p == nullptr: none
onecomp_status embedding_backward_run(onecomp_dtype dtype, const int32_t* tokens, int64_t n, const Rows& d_out, int64_t vocab, int64_t width, float scale,
                                      const Rows& base, const Rows& d_table, void* workspace, hipStream_t stream);

struct Loss {
    Rows h, weight, dh, dweight;
    const int32_t* targets;
    float *loss, *lse;                       // forward: results; gradients: lse as it was left
    const float *d_loss, *d_lse;
    int64_t tokens, width, vocab;
    float scale;
    void* workspace;
};
size_t loss_workspace_bytes(onecomp_dtype dtype, int64_t tokens, int64_t width, int64_t vocab, bool gradient);
onecomp_status loss_forward_run(onecomp_dtype dtype, const Loss& P, hipStream_t stream);
onecomp_status loss_backward_run(onecomp_dtype dtype, const Loss& P, hipStream_t stream);

}  // namespace token
}  // namespace onecomp
