// Launch interface of the feed-forward block's operators (norm, dropout, gated projections) between the C ABI and the kernels.
#ifndef RD_BLOCK_H_
#define RD_BLOCK_H_

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace rd {

// Which values dropout keeps, as a function of their place alone; border 0: all of them.
struct DropArgs {
    uint32_t border;          // a value stays where its 16 random bits are at least this
    float keep;               // what it is multiplied by then: 65536 / (65536 - border)
    uint64_t seed, offset;
    uint32_t first;           // number of the first row
};

struct NormArgs {
    const void *x, *residual, *weight;       // n x dim, n x dim or null, dim
    void *out, *sum;                         // n x dim, n x dim or null
    float *out_scale, *rstd;                 // n or null
    size_t x_stride, residual_stride, out_stride, sum_stride, n, dim;
    int dtype, sum_dtype, weight_dtype, out_dtype;      // rd_dtype_t
    float eps;
    DropArgs drop;
    cudaStream_t stream;
};

struct NormGradArgs {
    const void *grad_out, *sum, *weight, *grad_sum;     // grad_sum may be null
    const float *rstd;
    void *grad_x, *grad_residual, *grad_weight;         // each may be null
    size_t grad_out_stride, sum_stride, grad_sum_stride, grad_x_stride, grad_residual_stride, n, dim;
    int dtype, sum_dtype, weight_dtype;
    DropArgs drop;
    void *workspace;
    cudaStream_t stream;
};

struct DropoutArgs {
    const void *x;
    void *out;
    size_t x_stride, out_stride, n, dim;
    int dtype;
    DropArgs drop;
    cudaStream_t stream;
};

// Operands of the gated projections and of their gradient.
struct GatedArgs {
    const void *x, *gate_weight, *up_weight;            // n x dim, width x dim
    size_t x_stride, gate_weight_stride, up_weight_stride, n, dim, width;
    const float *x_scale, *gate_scale, *up_scale;       // 8 bits: n, width, width
    int dtype, out_dtype, activation;                   // rd_dtype_t, rd_activation_t
    void *out;                                          // n x width
    size_t out_stride;
    // what the projections give before the activation: written where not null, read by the gradient
    void *gate, *up;
    size_t gate_stride, up_stride;
    // gradient: outputs may be null
    const void *grad_out;
    void *grad_x, *grad_gate_weight, *grad_up_weight;
    size_t grad_out_stride, grad_x_stride, grad_gate_weight_stride, grad_up_weight_stride;
    void *workspace;
    cudaStream_t stream;
};

size_t gated_workspace(const GatedArgs &a);
cudaError_t gated_forward(const GatedArgs &a);
size_t gated_backward_workspace(const GatedArgs &a, bool want_x);
cudaError_t gated_backward(const GatedArgs &a);
// The word in which a kernel notes a wait that it gave up, cleared; block_status waits for the device first and covers both files.
cudaError_t norm_status(int *status);
cudaError_t block_status(int *status);

cudaError_t norm_forward(const NormArgs &a);
cudaError_t norm_backward(const NormGradArgs &a);
size_t norm_backward_workspace(size_t n, size_t dim);
cudaError_t dropout(const DropoutArgs &a);

}  // namespace rd

#endif  // RD_BLOCK_H_
