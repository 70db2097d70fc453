// The C ABI of the vocabulary operators (see include/rd.h): argument checking, then the launches.
#include <cuda_runtime.h>

#include <cmath>

#include "rd.h"
#include "rd_vocab.h"

using namespace rd;

namespace {

constexpr size_t kMostDim = 65536;
constexpr size_t kMostRows = (size_t(1) << 31) - 1024;       // rows and tokens are counted in 32 bits, with room for padding

bool is_float(int dtype) { return dtype == RD_FP32 || dtype == RD_BF16 || dtype == RD_FP16; }
size_t size_of(int dtype) { return dtype == RD_INT64 || dtype == RD_FP64 ? 8 : dtype == RD_BF16 || dtype == RD_FP16 ? 2 : 4; }
bool known(int dtype) { return dtype >= RD_INT32 && dtype <= RD_FP16; }
bool aligned(const void *p, size_t to) { return p && reinterpret_cast<uintptr_t>(p) % to == 0; }

// Memory that a call reads or writes: one run of bytes, or rows of `width` bytes that begin `stride` bytes apart.
struct Span {
    uintptr_t begin, end;
    size_t width, stride;     // stride 0: one run
    Span(const void *p, size_t bytes) : begin(reinterpret_cast<uintptr_t>(p)), end(p ? begin + bytes : begin), width(end - begin), stride(0) {}
    Span(const void *p, size_t rows, size_t row_stride, size_t dim, size_t esize) : Span(p, rows ? ((rows - 1) * row_stride + dim) * esize : 0)
    {
        if (p && rows > 1 && row_stride > dim) {
            width = dim * esize;
            stride = row_stride * esize;
        }
    }
    // Spans that lie apart do not meet, nor do columns side by side in rows of the same buffer, which are rows of the same stride (or
    // one run beside such rows).  Rows of different strides are taken to meet when their spans do.
    bool meets(const Span &o) const
    {
        if (begin >= o.end || o.begin >= end) return false;
        if (stride && o.stride && stride != o.stride) return true;
        const size_t s = stride ? stride : o.stride;
        if (!s) return true;
        const size_t at = o.begin >= begin ? (o.begin - begin) % s : (s - (begin - o.begin) % s) % s;       // where o's rows begin in this one's
        return at < width || at + o.width > s;
    }
};

// A matrix's stride: at least a row (0 for an input whose rows are all the same one), and the whole matrix within the address space.
bool stride_ok(size_t rows, size_t stride, size_t dim, size_t esize, bool may_repeat = false)
{
    return (stride >= dim || (may_repeat && stride == 0)) && (rows == 0 || stride <= (size_t(1) << 47) / esize / rows);
}

int status_of(cudaError_t e) { return e == cudaSuccess ? RD_OK : RD_ERR_CUDA; }

int check_vocab(const rd_vocab_t *v)
{
    if (!v) return RD_ERR_INVALID_ARG;
    if (!known(v->dtype) || (v->label_type != RD_INT32 && v->label_type != RD_INT64)) return RD_ERR_INVALID_ARG;
    if (v->dim < 1 || v->dim > kMostDim || v->rows < 1 || v->first_row < 0 || !std::isfinite(v->scale) || v->scale == 0.0f || !std::isfinite(v->z_loss)) return RD_ERR_INVALID_ARG;
    if (v->dtype != RD_BF16 && v->dtype != RD_FP16) return RD_ERR_UNSUPPORTED;
    if (v->rows > kMostRows || v->n > kMostRows) return RD_ERR_UNSUPPORTED;
    // output tiles are counted in 32 bits
    if ((v->n / 128 + 1) * (v->rows / 256 + 1) >= size_t(1) << 31 || (v->n / 128 + 1) * (v->dim / 256 + 1) >= size_t(1) << 24 ||
        (v->rows / 128 + 1) * (v->dim / 256 + 1) >= size_t(1) << 31)
        return RD_ERR_UNSUPPORTED;
    if (!aligned(v->weight, 2) || !stride_ok(v->rows, v->weight_stride, v->dim, 2)) return RD_ERR_INVALID_ARG;
    if (v->n && (!aligned(v->hidden, 2) || !stride_ok(v->n, v->hidden_stride, v->dim, 2, true) || !aligned(v->labels, size_of(v->label_type)))) return RD_ERR_INVALID_ARG;
    return RD_OK;
}

VocabArgs vocab_args(const rd_vocab_t *v)
{
    VocabArgs a{};
    a.hidden = v->hidden;
    a.hidden_stride = v->hidden_stride;
    a.weight = v->weight;
    a.weight_stride = v->weight_stride;
    a.labels = v->labels;
    a.n = v->n;
    a.rows = v->rows;
    a.dim = v->dim;
    a.first_row = v->first_row;
    a.scale = v->scale;
    a.z_loss = v->z_loss;
    a.bf16 = v->dtype == RD_BF16;
    a.wide_labels = v->label_type == RD_INT64;
    return a;
}

// Whether a written span meets one that is read, or another written one.
template <int W, int R> bool overlap(const Span (&written)[W], const Span (&read)[R])
{
    for (int i = 0; i < W; i++) {
        for (int j = 0; j < R; j++)
            if (written[i].meets(read[j])) return true;
        for (int j = 0; j < i; j++)
            if (written[i].meets(written[j])) return true;
    }
    return false;
}

}  // namespace

extern "C" {

int rd_embed(const void *d_table, size_t table_stride, size_t rows, size_t dim, rd_dtype_t dtype, const void *d_ids, rd_dtype_t id_type, size_t n, int64_t first_row,
             float scale, void *d_out, size_t out_stride, void *cuda_stream)
{
    if (!known(dtype) || (id_type != RD_INT32 && id_type != RD_INT64)) return RD_ERR_INVALID_ARG;
    if (dim < 1 || dim > kMostDim || rows < 1 || first_row < 0 || !std::isfinite(scale)) return RD_ERR_INVALID_ARG;
    if (!is_float(dtype) || rows > kMostRows || n > kMostRows) return RD_ERR_UNSUPPORTED;
    const size_t esize = size_of(dtype);
    if (!aligned(d_table, esize) || !stride_ok(rows, table_stride, dim, esize)) return RD_ERR_INVALID_ARG;
    if (n == 0) return RD_OK;
    if (!aligned(d_out, esize) || !stride_ok(n, out_stride, dim, esize) || !aligned(d_ids, size_of(id_type))) return RD_ERR_INVALID_ARG;
    const Span written[] = {Span(d_out, n, out_stride, dim, esize)};
    const Span read[] = {Span(d_table, rows, table_stride, dim, esize), Span(d_ids, n * size_of(id_type))};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    const EmbedArgs a{d_table, d_ids, d_out, table_stride, out_stride, rows, dim, n, first_row, scale, int(dtype), id_type == RD_INT64, static_cast<cudaStream_t>(cuda_stream)};
    return status_of(embed_forward(a));
}

int rd_embed_grad_workspace(size_t rows, size_t dim, size_t n, size_t *bytes)
{
    if (!bytes || dim < 1 || dim > kMostDim || rows < 1) return RD_ERR_INVALID_ARG;
    if (rows > kMostRows || n > kMostRows) return RD_ERR_UNSUPPORTED;
    *bytes = embed_backward_workspace(rows, dim, n);
    return RD_OK;
}

int rd_embed_grad(const void *d_grad_out, size_t grad_stride, rd_dtype_t dtype, const void *d_ids, rd_dtype_t id_type, size_t n, int64_t first_row, float scale,
                  void *d_grad_table, size_t table_stride, rd_dtype_t table_dtype, size_t rows, size_t dim, int accumulate, void *d_workspace, size_t workspace_bytes,
                  void *cuda_stream)
{
    if (!known(dtype) || !known(table_dtype) || (id_type != RD_INT32 && id_type != RD_INT64)) return RD_ERR_INVALID_ARG;
    if (dim < 1 || dim > kMostDim || rows < 1 || first_row < 0 || !std::isfinite(scale)) return RD_ERR_INVALID_ARG;
    if (!is_float(dtype) || (table_dtype != dtype && table_dtype != RD_FP32) || rows > kMostRows || n > kMostRows) return RD_ERR_UNSUPPORTED;
    const size_t esize = size_of(dtype), tsize = size_of(table_dtype);
    if (!aligned(d_grad_table, tsize) || !stride_ok(rows, table_stride, dim, tsize)) return RD_ERR_INVALID_ARG;
    if (n && (!aligned(d_grad_out, esize) || !stride_ok(n, grad_stride, dim, esize, true) || !aligned(d_ids, size_of(id_type)))) return RD_ERR_INVALID_ARG;
    if (!aligned(d_workspace, 256)) return RD_ERR_INVALID_ARG;
    const size_t need = embed_backward_workspace(rows, dim, n);
    if (workspace_bytes < need) return RD_ERR_TOO_SMALL;
    const Span written[] = {Span(d_grad_table, rows, table_stride, dim, tsize), Span(d_workspace, need)};
    const Span read[] = {Span(n ? d_grad_out : nullptr, n, grad_stride, dim, esize), Span(n ? d_ids : nullptr, n * size_of(id_type))};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    const EmbedGradArgs a{d_grad_out, d_ids, d_grad_table, grad_stride, table_stride, rows, dim, n, first_row, scale, int(dtype), int(table_dtype),
                          id_type == RD_INT64, accumulate != 0, d_workspace, static_cast<cudaStream_t>(cuda_stream)};
    return status_of(embed_backward(a));
}

int rd_vocab_loss_workspace(const rd_vocab_t *v, size_t *bytes)
{
    if (!bytes) return RD_ERR_INVALID_ARG;
    if (int rc = check_vocab(v)) return rc;
    *bytes = vocab_loss_workspace(vocab_args(v));
    return RD_OK;
}

int rd_vocab_loss(const rd_vocab_t *v, float *d_loss, float *d_lse, float *d_target, void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (int rc = check_vocab(v)) return rc;
    if (v->n == 0) return RD_OK;
    if (!d_loss && !d_lse && !d_target) return RD_ERR_INVALID_ARG;
    for (const float *p : {d_loss, d_lse, d_target})
        if (p && !aligned(p, 4)) return RD_ERR_INVALID_ARG;
    if (!aligned(d_workspace, 256)) return RD_ERR_INVALID_ARG;
    VocabArgs a = vocab_args(v);
    const size_t need = vocab_loss_workspace(a);
    if (workspace_bytes < need) return RD_ERR_TOO_SMALL;
    const Span written[] = {Span(d_loss, v->n * 4), Span(d_lse, v->n * 4), Span(d_target, v->n * 4), Span(d_workspace, need)};
    const Span read[] = {Span(v->hidden, v->n, v->hidden_stride, v->dim, 2), Span(v->weight, v->rows, v->weight_stride, v->dim, 2), Span(v->labels, v->n * size_of(v->label_type))};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    a.loss = d_loss;
    a.lse_out = d_lse;
    a.target = d_target;
    a.workspace = d_workspace;
    a.stream = static_cast<cudaStream_t>(cuda_stream);
    return status_of(vocab_loss(a));
}

int rd_vocab_loss_grad_workspace(const rd_vocab_t *v, int want_hidden, int want_weight, size_t *bytes)
{
    if (!bytes || (!want_hidden && !want_weight)) return RD_ERR_INVALID_ARG;
    if (int rc = check_vocab(v)) return rc;
    *bytes = vocab_loss_grad_workspace(vocab_args(v), want_hidden != 0);
    return RD_OK;
}

int rd_vocab_loss_grad(const rd_vocab_t *v, const float *d_lse, const float *d_grad_loss, size_t grad_loss_stride, void *d_grad_hidden, size_t grad_hidden_stride,
                       void *d_grad_weight, size_t grad_weight_stride, void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (int rc = check_vocab(v)) return rc;
    const size_t n = v->n;
    if (n && !d_grad_hidden && !d_grad_weight) return RD_ERR_INVALID_ARG;
    if (d_grad_hidden && (!aligned(d_grad_hidden, 2) || !stride_ok(n, grad_hidden_stride, v->dim, 2))) return RD_ERR_INVALID_ARG;
    if (d_grad_weight && (!aligned(d_grad_weight, 2) || !stride_ok(v->rows, grad_weight_stride, v->dim, 2))) return RD_ERR_INVALID_ARG;
    if (n == 0) {
        if (!d_grad_weight) return RD_OK;
        if (Span(d_grad_weight, v->rows, grad_weight_stride, v->dim, 2).meets(Span(v->weight, v->rows, v->weight_stride, v->dim, 2))) return RD_ERR_INVALID_ARG;
        return status_of(cudaMemset2DAsync(d_grad_weight, grad_weight_stride * 2, 0, v->dim * 2, v->rows, static_cast<cudaStream_t>(cuda_stream)));
    }
    if (!aligned(d_lse, 4) || !aligned(d_grad_loss, 4) || grad_loss_stride > (size_t(1) << 45) / n || !aligned(d_workspace, 256)) return RD_ERR_INVALID_ARG;
    VocabArgs a = vocab_args(v);
    a.grad_hidden = d_grad_hidden;
    const size_t need = vocab_loss_grad_workspace(a, d_grad_hidden != nullptr);
    if (workspace_bytes < need) return RD_ERR_TOO_SMALL;
    const Span written[] = {Span(d_grad_hidden, n, grad_hidden_stride, v->dim, 2), Span(d_grad_weight, v->rows, grad_weight_stride, v->dim, 2), Span(d_workspace, need)};
    const Span read[] = {Span(v->hidden, n, v->hidden_stride, v->dim, 2), Span(v->weight, v->rows, v->weight_stride, v->dim, 2),
                         Span(v->labels, n * size_of(v->label_type)), Span(d_lse, n * 4), Span(d_grad_loss, ((n - 1) * grad_loss_stride + 1) * 4)};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    a.lse = d_lse;
    a.grad_loss = d_grad_loss;
    a.grad_loss_stride = grad_loss_stride;
    a.grad_hidden_stride = grad_hidden_stride;
    a.grad_weight = d_grad_weight;
    a.grad_weight_stride = grad_weight_stride;
    a.workspace = d_workspace;
    a.stream = static_cast<cudaStream_t>(cuda_stream);
    return status_of(vocab_loss_grad(a));
}

int rd_vocab_status(int *device_status)
{
    if (!device_status) return RD_ERR_INVALID_ARG;
    int s = 0;
    if (vocab_status(&s) != cudaSuccess) return RD_ERR_CUDA;
    *device_status = s ? RD_ERR_TIMEOUT : RD_OK;
    return RD_OK;
}

}  // extern "C"
