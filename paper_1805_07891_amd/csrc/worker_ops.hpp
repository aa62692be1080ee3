// The worker's operators: what the C interface (worker_api.cpp) and the
// kernels (layer_norm.hip, vocab_loss.hip) share.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

namespace phub {

// Element types of hidden states (phub_type of the C interface).
enum ElemType { kF32 = 0, kBf16 = 1, kF16 = 2 };

// ------------------------------------------------------------- layer norm

struct NormArgs {
    int type;
    int64_t rows, cols;
    const void* x;
    int64_t x_stride;  // elements between rows, here and below
    const void* dy;
    int64_t dy_stride;
    const float* weight;  // null: ones
    const float* bias;    // null: zeros
    float eps;
    void* y;  // forward: y; backward: dx (null: not wanted)
    int64_t y_stride;
    float* mean;  // forward: may be null
    float* rstd;
    float* dweight;  // backward: may be null
    float* dbias;
    bool accumulate;
    float* partial;  // backward: 2 * norm_strips(rows, cols) * cols floats
};

// Rows of partial sums that the backward pass leaves for each of the two
// gradients.
int64_t norm_strips(int64_t rows, int64_t cols);
hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream);
hipError_t launch_layer_norm_grad(const NormArgs& a, hipStream_t stream);

// ------------------------------------- losses over a vocabulary's products

struct VocabArgs {
    int type;
    int64_t rows, cols, vocab;
    const void* x;
    int64_t x_stride;
    const void* w;
    int64_t w_stride;
    int top;                // teacher's entries a row; 0: targets
    const int64_t* target;  // [rows], or the teacher's indices, [rows][top]
    const float* logit;     // teacher's logits, [rows][top]
    float temperature;      // 1 for targets
    float* loss;            // forward
    float* lse;             // forward: written; backward: read
    const float* dloss;     // backward; null: ones
    void* dx;               // may be null
    int64_t dx_stride;
    float* dw;              // may be null
    int64_t dw_stride;
    bool accumulate;
};

// Bytes of workspace: the fewest that a call takes and as many as it has use for.  Only the
// sizes, strides and the alignment of x and w count.
void vocab_bytes(const VocabArgs& a, bool grad, int64_t* least, int64_t* best);
// Vocabulary rows of the largest pieces that so many bytes are enough for; 0: too few.
int64_t vocab_piece(const VocabArgs& a, bool grad, int64_t bytes);
// piece: from vocab_piece; workspace: 256-byte aligned.
hipError_t launch_vocab_loss(const VocabArgs& a, int64_t piece, void* workspace, hipStream_t stream);
// (no rows: neither piece nor workspace count)
hipError_t launch_vocab_loss_grad(const VocabArgs& a, int64_t piece, void* workspace,
                                  hipStream_t stream);

}  // namespace phub
