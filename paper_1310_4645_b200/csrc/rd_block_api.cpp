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

constexpr size_t kMostWidth = size_t(1) << 20;

int check_gated(const rd_gated_t *v)
{
    if (!v || (!known(v->dtype) && v->dtype != RD_E4M3) || int(v->activation) < RD_SILU || int(v->activation) > RD_RELU) return RD_ERR_INVALID_ARG;
    if (v->dim < 1 || v->dim > kMostDim || v->width < 1) return RD_ERR_INVALID_ARG;
    const bool eight = v->dtype == RD_E4M3;
    if (!eight && v->dtype != RD_BF16 && v->dtype != RD_FP16) return RD_ERR_UNSUPPORTED;
    if (v->n > kMostRows || v->width > kMostWidth) return RD_ERR_UNSUPPORTED;
    // output tiles are counted in 32 bits
    if ((v->n / 128 + 1) * (v->width / 16 + 1) >= size_t(1) << 31 || (v->n / 128 + 1) * (v->dim / 256 + 1) >= size_t(1) << 24) return RD_ERR_UNSUPPORTED;
    const size_t esize = eight ? 1 : 2;
    for (const void *w : {v->gate_weight, v->up_weight})
        if (!aligned(w, esize)) return RD_ERR_INVALID_ARG;
    if (!stride_ok(v->width, v->gate_weight_stride, v->dim, esize) || !stride_ok(v->width, v->up_weight_stride, v->dim, esize)) return RD_ERR_INVALID_ARG;
    if (v->n && (!aligned(v->x, esize) || !stride_ok(v->n, v->x_stride, v->dim, esize, true))) return RD_ERR_INVALID_ARG;
    for (const float *s : {v->x_scale, v->gate_scale, v->up_scale})
        if (eight ? (v->n && !aligned(s, 4)) : s != nullptr) return RD_ERR_INVALID_ARG;
    return RD_OK;
}

GatedArgs gated_args(const rd_gated_t *v)
{
    GatedArgs a{};
    a.x = v->x;
    a.x_stride = v->x_stride;
    a.gate_weight = v->gate_weight;
    a.gate_weight_stride = v->gate_weight_stride;
    a.up_weight = v->up_weight;
    a.up_weight_stride = v->up_weight_stride;
    a.x_scale = v->x_scale;
    a.gate_scale = v->gate_scale;
    a.up_scale = v->up_scale;
    a.n = v->n;
    a.dim = v->dim;
    a.width = v->width;
    a.dtype = int(v->dtype);
    a.activation = int(v->activation);
    return a;
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

int rd_gated_workspace(const rd_gated_t *v, size_t *bytes)
{
    if (!bytes) return RD_ERR_INVALID_ARG;
    if (int rc = check_gated(v)) return rc;
    *bytes = gated_workspace(gated_args(v));
    return RD_OK;
}

int rd_gated(const rd_gated_t *v, void *d_out, size_t out_stride, rd_dtype_t out_dtype, void *d_gate, size_t gate_stride, void *d_up, size_t up_stride, void *d_workspace,
             size_t workspace_bytes, void *cuda_stream)
{
    if (int rc = check_gated(v)) return rc;
    if (!known(out_dtype) && out_dtype != RD_E4M3) return RD_ERR_INVALID_ARG;
    const bool eight = v->dtype == RD_E4M3;
    if (eight ? out_dtype != RD_BF16 && out_dtype != RD_FP16 : out_dtype != v->dtype) return RD_ERR_UNSUPPORTED;
    if (v->n == 0) return RD_OK;
    const size_t n = v->n, dim = v->dim, width = v->width, esize = eight ? 1 : 2;
    const Rows out{d_out, out_stride, n, width, 2}, gate{d_gate, gate_stride, n, width, 2}, up{d_up, up_stride, n, width, 2};
    if (!out.ok(false) || (gate.p && !gate.ok(false)) || (up.p && !up.ok(false))) return RD_ERR_INVALID_ARG;
    GatedArgs a = gated_args(v);
    const size_t need = gated_workspace(a);
    if (need && !aligned(d_workspace, 256)) return RD_ERR_INVALID_ARG;
    if (workspace_bytes < need) return RD_ERR_TOO_SMALL;
    const Span written[] = {out.span(), gate.span(), up.span(), Span(need ? d_workspace : nullptr, need)};
    const Span read[] = {Span(v->x, n, v->x_stride, dim, esize), Span(v->gate_weight, width, v->gate_weight_stride, dim, esize),
                         Span(v->up_weight, width, v->up_weight_stride, dim, esize), Span(v->x_scale, n * 4), Span(v->gate_scale, width * 4), Span(v->up_scale, width * 4)};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    a.out = d_out;
    a.out_stride = out_stride;
    a.out_dtype = int(out_dtype);
    a.gate = d_gate;
    a.gate_stride = gate_stride;
    a.up = d_up;
    a.up_stride = up_stride;
    a.workspace = d_workspace;
    a.stream = static_cast<cudaStream_t>(cuda_stream);
    return status_of(gated_forward(a));
}

int rd_gated_grad_workspace(const rd_gated_t *v, int want_x, size_t *bytes)
{
    if (!bytes) return RD_ERR_INVALID_ARG;
    if (int rc = check_gated(v)) return rc;
    if (v->dtype == RD_E4M3) return RD_ERR_UNSUPPORTED;
    *bytes = gated_backward_workspace(gated_args(v), want_x != 0);
    return RD_OK;
}

int rd_gated_grad(const rd_gated_t *v, const void *d_grad_out, size_t grad_out_stride, const void *d_gate, size_t gate_stride, const void *d_up, size_t up_stride, void *d_grad_x,
                  size_t grad_x_stride, void *d_grad_gate_weight, size_t grad_gate_weight_stride, void *d_grad_up_weight, size_t grad_up_weight_stride, void *d_workspace,
                  size_t workspace_bytes, void *cuda_stream)
{
    if (int rc = check_gated(v)) return rc;
    if (v->dtype == RD_E4M3) return RD_ERR_UNSUPPORTED;
    if (!d_grad_x && !d_grad_gate_weight && !d_grad_up_weight) return RD_ERR_INVALID_ARG;
    const size_t n = v->n, dim = v->dim, width = v->width;
    const Rows up_grad{d_grad_out, grad_out_stride, n, width, 2}, gate{d_gate, gate_stride, n, width, 2}, up{d_up, up_stride, n, width, 2};
    const Rows gx{d_grad_x, grad_x_stride, n, dim, 2}, gg{d_grad_gate_weight, grad_gate_weight_stride, width, dim, 2}, gu{d_grad_up_weight, grad_up_weight_stride, width, dim, 2};
    for (const Rows *r : {&gx, &gg, &gu})
        if (r->p && r->n && !r->ok(false)) return RD_ERR_INVALID_ARG;
    if (n && (!up_grad.ok(true) || !gate.ok(true) || !up.ok(true))) return RD_ERR_INVALID_ARG;
    GatedArgs a = gated_args(v);
    const size_t need = gated_backward_workspace(a, d_grad_x != nullptr);
    if (need && !aligned(d_workspace, 256)) return RD_ERR_INVALID_ARG;
    if (workspace_bytes < need) return RD_ERR_TOO_SMALL;
    auto of = [&](const Rows &r) { return Span(n ? r.p : nullptr, r.n, r.stride, r.dim, r.esize); };
    const Span written[] = {of(gx), gg.span(), gu.span(), Span(need ? d_workspace : nullptr, need)};
    const Span read[] = {Span(n ? v->x : nullptr, n, v->x_stride, dim, 2), Span(v->gate_weight, width, v->gate_weight_stride, dim, 2),
                         Span(v->up_weight, width, v->up_weight_stride, dim, 2), of(up_grad), of(gate), of(up)};
    if (overlap(written, read)) return RD_ERR_INVALID_ARG;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (n == 0) {
        for (const Rows *r : {&gg, &gu})
            if (r->p)
                if (const cudaError_t e = cudaMemset2DAsync(const_cast<void *>(r->p), r->stride * 2, 0, dim * 2, width, stream); e != cudaSuccess) return status_of(e);
        return RD_OK;
    }
    a.grad_out = d_grad_out;
    a.grad_out_stride = grad_out_stride;
    a.gate = const_cast<void *>(d_gate);
    a.gate_stride = gate_stride;
    a.up = const_cast<void *>(d_up);
    a.up_stride = up_stride;
    a.grad_x = d_grad_x;
    a.grad_x_stride = grad_x_stride;
    a.grad_gate_weight = d_grad_gate_weight;
    a.grad_gate_weight_stride = grad_gate_weight_stride;
    a.grad_up_weight = d_grad_up_weight;
    a.grad_up_weight_stride = grad_up_weight_stride;
    a.workspace = d_workspace;
    a.stream = stream;
    return status_of(gated_backward(a));
}

int rd_block_status(int *device_status)
{
    if (!device_status) return RD_ERR_INVALID_ARG;
    int s = 0;
    if (block_status(&s) != cudaSuccess) return RD_ERR_CUDA;
    *device_status = s ? RD_ERR_TIMEOUT : RD_OK;
    return RD_OK;
}

}  // extern "C"
