// Launch interface of the vocabulary operators (embedding, softmax cross entropy) between the C ABI and the kernels.
#ifndef RD_VOCAB_H_
#define RD_VOCAB_H_

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace rd {

struct EmbedArgs {
    const void *table;        // rows x dim, row stride in elements
    const void *ids;          // n token ids, 4 or 8 bytes each
    void *out;                // n x dim
    size_t table_stride, out_stride, rows, dim, n;
    long long first_row;      // id of the table's first row
    float scale;
    int dtype;                // rd_dtype_t
    bool wide_ids;            // 8-byte ids
    cudaStream_t stream;
};

struct EmbedGradArgs {
    const void *grad;         // n x dim
    const void *ids;
    void *table;              // rows x dim
    size_t grad_stride, table_stride, rows, dim, n;
    long long first_row;
    float scale;
    int dtype, table_dtype;
    bool wide_ids, accumulate;
    void *workspace;
    cudaStream_t stream;
};

// Operands of the loss and of its gradient.
struct VocabArgs {
    const void *hidden;       // n x dim
    const void *weight;       // rows x dim
    const void *labels;       // n, 4 or 8 bytes each
    size_t hidden_stride, weight_stride, n, rows, dim;
    long long first_row;
    float scale, z_loss;
    bool bf16, wide_labels;
    void *workspace;
    cudaStream_t stream;
    // loss: outputs (each may be null); gradient: lse is an input
    float *loss, *lse_out, *target;
    // gradient
    const float *lse, *grad_loss;
    size_t grad_loss_stride;  // 0: one value for all tokens
    void *grad_hidden, *grad_weight;
    size_t grad_hidden_stride, grad_weight_stride;
};

cudaError_t embed_forward(const EmbedArgs &a);
cudaError_t embed_backward(const EmbedGradArgs &a);
size_t embed_backward_workspace(size_t rows, size_t dim, size_t n);
size_t vocab_loss_workspace(const VocabArgs &a);
cudaError_t vocab_loss(const VocabArgs &a);
size_t vocab_loss_grad_workspace(const VocabArgs &a, bool want_hidden);
cudaError_t vocab_loss_grad(const VocabArgs &a);
// The word in which a kernel notes a wait that it gave up, cleared; vocab_status waits for the device first and covers both files.
cudaError_t embed_status(int *status);
cudaError_t vocab_status(int *status);

}  // namespace rd

#endif  // RD_VOCAB_H_
