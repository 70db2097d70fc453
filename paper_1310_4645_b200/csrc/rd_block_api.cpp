// The C ABI of the feed-forward block's operators (see include/rd.h): argument checking, then the launches.
#include <cuda_runtime.h>

#include <cmath>

#include "rd.h"
#include "rd_block.h"
#include "rd_checks.h"

using namespace rd;

namespace {

// A matrix of n rows that a call reads or writes.
struct Rows {
    const void *p;
    size_t stride, n, dim, esize;
    Span span() const { return Span(p, n, stride, dim, esize); }
    // exactly the same elements in the same places
    bool same(const Rows &o) const { return p == o.p && esize == o.esize && (stride == o.stride || n == 1); }
    bool ok(bool may_repeat) const { return aligned(p, esize) && stride_ok(n, stride, dim, esize, may_repeat); }
};

// Whether a written matrix meets a read one other than by being the same.
bool spoils(const Rows &written, const Rows &read) { return written.p && read.p && !written.same(read) && written.span().meets(read.span()); }

int drop_args(float drop, uint64_t seed, uint64_t offset, size_t first_row, size_t n, DropArgs *d)
{
    if (!(drop >= 0.0f && drop < 1.0f)) return RD_ERR_INVALID_ARG;
    const long border = std::lrint(double(drop) * 65536.0);
    if (border == 65536) return RD_ERR_INVALID_ARG;
    if (border && (first_row > (size_t(1) << 32) || first_row + n > size_t(1) << 32)) return RD_ERR_UNSUPPORTED;
    *d = DropArgs{uint32_t(border), float(65536.0 / double(65536 - border)), seed, offset, uint32_t(first_row)};
    return RD_OK;
}

// The types of rows, residual and weight, and the sizes.
int check_rows(int dtype, int sum_dtype, int weight_dtype, size_t n, size_t dim)
{
    for (const int t : {dtype, sum_dtype, weight_dtype})
        if (!known(t) && t != RD_E4M3) return RD_ERR_INVALID_ARG;
    if (dim < 1 || dim > kMostDim) return RD_ERR_INVALID_ARG;
    if (!is_float(dtype) || (sum_dtype != dtype && sum_dtype != RD_FP32) || (weight_dtype != dtype && weight_dtype != RD_FP32) || n > kMostRows) return RD_ERR_UNSUPPORTED;
    return RD_OK;
}

}  // namespace

extern "C" {

int rd_norm(const rd_norm_t *v, void *d_out, size_t out_stride, rd_dtype_t out_dtype, float *d_out_scale, void *d_sum, size_t sum_stride, float *d_rstd, void *cuda_stream)
{
    if (!v || (!known(out_dtype) && out_dtype != RD_E4M3) || !std::isfinite(v->eps) || v->eps < 0.0f) return RD_ERR_INVALID_ARG;
    if (int rc = check_rows(v->dtype, v->sum_dtype, v->weight_dtype, v->n, v->dim)) return rc;
    const bool eight = out_dtype == RD_E4M3;
    if (!eight && out_dtype != v->dtype) return RD_ERR_UNSUPPORTED;
    DropArgs drop;
    if (int rc = drop_args(v->drop, v->seed, v->offset, v->first_row, v->n, &drop)) return rc;
    const size_t n = v->n, dim = v->dim, esize = size_of(v->dtype), ssize = size_of(v->sum_dtype);
    if (!aligned(v->weight, size_of(v->weight_dtype))) return RD_ERR_INVALID_ARG;
    if (n == 0) return RD_OK;
    if (eight != (d_out_scale != nullptr)) return RD_ERR_INVALID_ARG;
    const Rows x{v->x, v->x_stride, n, dim, esize}, residual{v->residual, v->residual_stride, n, dim, ssize};
    const Rows out{d_out, out_stride, n, dim, eight ? 1 : esize}, sum{d_sum, sum_stride, n, dim, ssize};
    if (!x.ok(true) || (residual.p && !residual.ok(true)) || !out.ok(false) || (sum.p && !sum.ok(false))) return RD_ERR_INVALID_ARG;
    for (const float *p : {d_out_scale, d_rstd})
        if (p && !aligned(p, 4)) return RD_ERR_INVALID_ARG;
    const Span weight(v->weight, dim * size_of(v->weight_dtype)), scales(d_out_scale, n * 4), rstds(d_rstd, n * 4);
    for (const Rows *w : {&out, &sum})
        if (spoils(*w, x) || (residual.p && spoils(*w, residual)) || (w->p && w->span().meets(weight))) return RD_ERR_INVALID_ARG;
    const Span written[] = {out.span(), sum.span(), scales, rstds};
    const Span read[] = {weight};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    for (const Span &w : {scales, rstds})
        if (w.meets(x.span()) || w.meets(residual.span())) return RD_ERR_INVALID_ARG;
    const NormArgs a{v->x, v->residual, v->weight, d_out, d_sum, d_out_scale, d_rstd, x.stride, residual.stride, out_stride, sum_stride, n, dim,
                     int(v->dtype), int(v->sum_dtype), int(v->weight_dtype), int(out_dtype), v->eps, drop, static_cast<cudaStream_t>(cuda_stream)};
    return status_of(norm_forward(a));
}

int rd_norm_grad_workspace(size_t n, size_t dim, size_t *bytes)
{
    if (!bytes || dim < 1 || dim > kMostDim) return RD_ERR_INVALID_ARG;
    if (n > kMostRows) return RD_ERR_UNSUPPORTED;
    *bytes = norm_backward_workspace(n, dim);
    return RD_OK;
}

int rd_norm_grad(const rd_norm_grad_t *v, void *d_grad_x, size_t grad_x_stride, void *d_grad_residual, size_t grad_residual_stride, void *d_grad_weight, void *d_workspace,
                 size_t workspace_bytes, void *cuda_stream)
{
    if (!v) return RD_ERR_INVALID_ARG;
    if (int rc = check_rows(v->dtype, v->sum_dtype, v->weight_dtype, v->n, v->dim)) return rc;
    DropArgs drop;
    if (int rc = drop_args(v->drop, v->seed, v->offset, v->first_row, v->n, &drop)) return rc;
    const size_t n = v->n, dim = v->dim, esize = size_of(v->dtype), ssize = size_of(v->sum_dtype), wsize = size_of(v->weight_dtype);
    if (!d_grad_x && !d_grad_residual && !d_grad_weight) return RD_ERR_INVALID_ARG;
    if (!aligned(v->weight, wsize) || (d_grad_weight && !aligned(d_grad_weight, wsize))) return RD_ERR_INVALID_ARG;
    const Rows up{v->grad_out, v->grad_out_stride, n, dim, esize}, sum{v->sum, v->sum_stride, n, dim, ssize}, more{v->grad_sum, v->grad_sum_stride, n, dim, ssize};
    const Rows gx{d_grad_x, grad_x_stride, n, dim, esize}, gr{d_grad_residual, grad_residual_stride, n, dim, ssize};
    const size_t need = d_grad_weight ? norm_backward_workspace(n, dim) : 0;
    if (need && !aligned(d_workspace, 256)) return RD_ERR_INVALID_ARG;
    if (workspace_bytes < need) return RD_ERR_TOO_SMALL;
    const Span weight(v->weight, dim * wsize), grad_weight(d_grad_weight, dim * wsize), workspace(need ? d_workspace : nullptr, need), rstd(n ? v->rstd : nullptr, n * 4);
    if (n) {
        if (!up.ok(true) || !sum.ok(true) || (more.p && !more.ok(true)) || !aligned(v->rstd, 4) || (gx.p && !gx.ok(false)) || (gr.p && !gr.ok(false))) return RD_ERR_INVALID_ARG;
        for (const Rows *w : {&gx, &gr})
            for (const Rows *r : {&up, &sum, &more})
                if (spoils(*w, *r)) return RD_ERR_INVALID_ARG;
        const Span written[] = {gx.span(), gr.span(), grad_weight, workspace};
        const Span read[] = {weight, rstd};
        if (overlap(written, read)) return RD_ERR_INVALID_ARG;
        for (const Span &w : {grad_weight, workspace})
            for (const Rows *r : {&up, &sum, &more})
                if (r->p && w.meets(r->span())) return RD_ERR_INVALID_ARG;
    } else if (!d_grad_weight) {
        return RD_OK;
    } else if (grad_weight.meets(weight)) {
        return RD_ERR_INVALID_ARG;
    }
    const NormGradArgs a{v->grad_out, v->sum, v->weight, v->grad_sum, v->rstd, d_grad_x, d_grad_residual, d_grad_weight, up.stride, sum.stride, more.stride, grad_x_stride,
                         grad_residual_stride, n, dim, int(v->dtype), int(v->sum_dtype), int(v->weight_dtype), drop, d_workspace, static_cast<cudaStream_t>(cuda_stream)};
    return status_of(norm_backward(a));
}

int rd_dropout(const void *d_x, size_t x_stride, size_t n, size_t dim, rd_dtype_t dtype, float drop, uint64_t seed, uint64_t offset, size_t first_row, void *d_out,
               size_t out_stride, void *cuda_stream)
{
    if (int rc = check_rows(dtype, dtype, dtype, n, dim)) return rc;
    DropArgs d;
    if (int rc = drop_args(drop, seed, offset, first_row, n, &d)) return rc;
    if (n == 0) return RD_OK;
    const Rows x{d_x, x_stride, n, dim, size_of(dtype)}, out{d_out, out_stride, n, dim, size_of(dtype)};
    if (!x.ok(true) || !out.ok(false) || spoils(out, x)) return RD_ERR_INVALID_ARG;
    const DropoutArgs a{d_x, d_out, x_stride, out_stride, n, dim, int(dtype), d, static_cast<cudaStream_t>(cuda_stream)};
    return status_of(dropout(a));
}

}  // extern "C"
