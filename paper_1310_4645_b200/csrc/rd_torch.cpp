// Marshalling of the operators' tensors (vocabulary, feed-forward block): the same checks and calls that ctypes would make, without the interpreter.
// A call on one token takes some 3 microseconds on the device; reading its tensors' properties, allocating and calling from Python
// took 9 to 17 on the host (passes back to back: rd_embed of one token 8.4 us with ctypes, 3.7 with this; rd_embed_grad of 257 tokens
// 16.3, 10.4).  Nothing is computed here.
//
// Every function returns its result, or the negative rd_status_t of the call as an int; wrong tensors raise ValueError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <new>
#include <stdexcept>

#include "rd.h"

namespace {

struct PythonError {};            // an exception that Python already knows

[[noreturn]] void wrong(const char *what)
{
    PyErr_SetString(PyExc_ValueError, what);
    throw PythonError();
}

const at::Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) wrong(what);
    return THPVariable_Unpack(o);
}

rd_dtype_t code(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kInt: return RD_INT32;
    case at::kFloat: return RD_FP32;
    case at::kLong: return RD_INT64;
    case at::kDouble: return RD_FP64;
    case at::kBFloat16: return RD_BF16;
    case at::kHalf: return RD_FP16;
    case at::kFloat8_e4m3fn: return RD_E4M3;
    default: break;
    }
    PyErr_SetString(PyExc_TypeError, "int32, float32, int64, float64, bfloat16, float16 or float8_e4m3fn expected");
    throw PythonError();
}

// A 2-D CUDA tensor whose rows are contiguous.
struct Matrix {
    void *data;
    size_t stride, rows, dim;
    Matrix(const at::Tensor &t, const char *what)
    {
        if (!t.is_cuda() || t.dim() != 2) wrong(what);
        const auto size = t.sizes(), strides = t.strides();
        if (strides[1] != 1 && size[1] > 1) wrong(what);
        data = t.data_ptr();
        rows = size_t(size[0]);
        dim = size_t(size[1]);
        stride = rows > 1 ? size_t(strides[0]) : dim;
    }
};

void *vector(const at::Tensor &t, size_t n, c10::Device device, const char *what)
{
    if (t.device() != device || t.dim() != 1 || size_t(t.size(0)) != n || !t.is_contiguous()) wrong(what);
    return t.data_ptr();
}

void like(const at::Tensor &t, const at::Tensor &operand)
{
    if (t.sizes() != operand.sizes() || t.scalar_type() != operand.scalar_type() || t.device() != operand.device())
        wrong("a gradient or out has its operand's shape, dtype and device");
}

int64_t whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    return v;
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return float(v);
}

at::Tensor empty(c10::IntArrayRef size, at::ScalarType type, c10::Device device) { return at::detail::empty_cuda(size, type, device, c10::nullopt); }

// Temporary memory: the caller's tensor, or the allocator's, given back (in the stream's order) as soon as the call is enqueued.
struct Workspace {
    void *data = nullptr;
    size_t size = 0;
    bool own = false;
    Workspace(PyObject *given, size_t need, c10::Device device, cudaStream_t stream)
    {
        if (given != Py_None) {
            const at::Tensor &t = tensor(given, "workspace must be a CUDA tensor");
            if (t.device() != device || !t.is_contiguous()) wrong("workspace must be a contiguous CUDA tensor on the operands' device");
            data = t.data_ptr();
            size = t.nbytes();
        } else if (need) {
            data = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(need, stream);
            size = need;
            own = true;
        }
    }
    ~Workspace()
    {
        if (own) c10::cuda::CUDACachingAllocator::raw_delete(data);
    }
    Workspace(const Workspace &) = delete;
    Workspace &operator=(const Workspace &) = delete;
};

PyObject *status(int rc) { return PyLong_FromLong(rc); }

// Runs f, turning C++ exceptions into Python's.
template <typename F> PyObject *guarded(Py_ssize_t given, Py_ssize_t wanted, F &&f)
{
    if (given != wanted) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", wanted, given);
        return nullptr;
    }
    try {
        return f();
    } catch (const PythonError &) {
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

template <typename F> int without_gil(F &&f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = f();
    Py_END_ALLOW_THREADS return rc;
}

// table, ids, out, first_row, scale
PyObject *embed(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 5, [&]() -> PyObject * {
        const at::Tensor &table = tensor(a[0], "table must be a 2-D CUDA tensor"), &ids = tensor(a[1], "ids must be a CUDA vector");
        const Matrix t(table, "table must be a 2-D CUDA tensor with contiguous rows");
        const c10::cuda::OptionalCUDAGuard guard(table.device());
        const size_t n = size_t(ids.numel());
        const void *at_ids = vector(ids, n, table.device(), "ids must be a contiguous CUDA vector on the table's device");
        const bool fresh = a[2] == Py_None;
        const at::Tensor out = fresh ? empty({int64_t(n), int64_t(t.dim)}, table.scalar_type(), table.device()) : tensor(a[2], "out must be a 2-D CUDA tensor");
        const Matrix o(out, "out must be a 2-D CUDA tensor with contiguous rows");
        if (o.rows != n || o.dim != t.dim || out.scalar_type() != table.scalar_type() || out.device() != table.device())
            wrong("out must be [n, dim] with table's dtype and device");
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(table.device().index());
        const int64_t first = whole(a[3]);
        const float scale = real(a[4]);
        const rd_dtype_t dtype = code(table), id_type = code(ids);
        const int rc = without_gil([&] { return rd_embed(t.data, t.stride, t.rows, t.dim, dtype, at_ids, id_type, n, first, scale, o.data, o.stride, stream); });
        if (rc != RD_OK) return status(rc);
        return fresh ? THPVariable_Wrap(out) : Py_NewRef(a[2]);
    });
}

// grad_out, ids, grad_table, first_row, scale, accumulate, workspace
PyObject *embed_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 7, [&]() -> PyObject * {
        const at::Tensor &grad = tensor(a[0], "grad_out must be a 2-D CUDA tensor"), &ids = tensor(a[1], "ids must be a CUDA vector");
        const at::Tensor &table = tensor(a[2], "grad_table must be a 2-D CUDA tensor");
        const Matrix g(grad, "grad_out must be a 2-D CUDA tensor with contiguous rows"), t(table, "grad_table must be a 2-D CUDA tensor with contiguous rows");
        const c10::cuda::OptionalCUDAGuard guard(grad.device());
        const void *at_ids = vector(ids, g.rows, grad.device(), "ids must be a contiguous CUDA vector with one value per token, on the operands' device");
        if (t.dim != g.dim || table.device() != grad.device()) wrong("grad_table must be [rows, dim] on grad_out's device");
        const int64_t first = whole(a[3]);
        const float scale = real(a[4]);
        const int accumulate = PyObject_IsTrue(a[5]);
        if (accumulate < 0) throw PythonError();
        const rd_dtype_t dtype = code(grad), id_type = code(ids), table_dtype = code(table);
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(grad.device().index());
        size_t need = 0;
        if (const int rc = rd_embed_grad_workspace(t.rows, t.dim, g.rows, &need)) return status(rc);
        const Workspace w(a[6], need, grad.device(), stream);
        const int rc = without_gil([&] {
            return rd_embed_grad(g.data, g.stride, dtype, at_ids, id_type, g.rows, first, scale, t.data, t.stride, table_dtype, t.rows, t.dim, accumulate, w.data, w.size, stream);
        });
        return rc != RD_OK ? status(rc) : Py_NewRef(a[2]);
    });
}

// hidden, weight, labels
rd_vocab_t operands(PyObject *const *a, const at::Tensor &hidden, const at::Tensor &weight, const at::Tensor &labels)
{
    const Matrix h(hidden, "hidden must be a 2-D CUDA tensor with contiguous rows"), w(weight, "weight must be a 2-D CUDA tensor with contiguous rows");
    if (w.dim != h.dim || weight.scalar_type() != hidden.scalar_type() || weight.device() != hidden.device())
        wrong("weight must be [rows, dim] with hidden's dtype and device");
    rd_vocab_t v;
    v.hidden = h.data;
    v.hidden_stride = h.stride;
    v.weight = w.data;
    v.weight_stride = w.stride;
    v.labels = vector(labels, h.rows, hidden.device(), "labels must be a contiguous CUDA vector with one value per token, on the operands' device");
    v.n = h.rows;
    v.rows = w.rows;
    v.dim = h.dim;
    v.first_row = whole(a[0]);
    v.dtype = code(hidden);
    v.label_type = code(labels);
    v.scale = real(a[1]);
    v.z_loss = real(a[2]);
    return v;
}

// hidden, weight, labels, first_row, scale, z_loss, workspace
PyObject *vocab_loss(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 7, [&]() -> PyObject * {
        const at::Tensor &hidden = tensor(a[0], "hidden must be a 2-D CUDA tensor"), &weight = tensor(a[1], "weight must be a 2-D CUDA tensor");
        const rd_vocab_t v = operands(a + 3, hidden, weight, tensor(a[2], "labels must be a CUDA vector"));
        const c10::cuda::OptionalCUDAGuard guard(hidden.device());
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(hidden.device().index());
        size_t need = 0;
        if (const int rc = rd_vocab_loss_workspace(&v, &need)) return status(rc);
        at::Tensor out[3];
        for (at::Tensor &t : out) t = empty({int64_t(v.n)}, at::kFloat, hidden.device());
        const Workspace w(a[6], need, hidden.device(), stream);
        float *p[3] = {static_cast<float *>(out[0].data_ptr()), static_cast<float *>(out[1].data_ptr()), static_cast<float *>(out[2].data_ptr())};
        const int rc = without_gil([&] { return rd_vocab_loss(&v, p[0], p[1], p[2], w.data, w.size, stream); });
        if (rc != RD_OK) return status(rc);
        PyObject *r = PyTuple_New(3);
        if (!r) throw PythonError();
        for (int k = 0; k < 3; k++) PyTuple_SET_ITEM(r, k, THPVariable_Wrap(std::move(out[k])));
        return r;
    });
}

// hidden, weight, labels, first_row, scale, z_loss, workspace, lse, grad_loss, grad_hidden, grad_weight
PyObject *vocab_loss_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&]() -> PyObject * {
        const at::Tensor &hidden = tensor(a[0], "hidden must be a 2-D CUDA tensor"), &weight = tensor(a[1], "weight must be a 2-D CUDA tensor");
        const rd_vocab_t v = operands(a + 3, hidden, weight, tensor(a[2], "labels must be a CUDA vector"));
        const c10::cuda::OptionalCUDAGuard guard(hidden.device());
        const at::Tensor &lse = tensor(a[7], "lse must be a CUDA vector"), &up = tensor(a[8], "grad_loss must be a CUDA tensor");
        const void *at_lse = vector(lse, v.n, hidden.device(), "lse must be a contiguous CUDA vector with one value per token, on the operands' device");
        if (up.device() != hidden.device() || up.dim() > 1 || (up.dim() == 1 && size_t(up.size(0)) != v.n) || up.scalar_type() != at::kFloat ||
            lse.scalar_type() != at::kFloat)
            wrong("lse and grad_loss must be float32 CUDA vectors with one value per token");
        const size_t up_stride = up.dim() == 0 ? 0 : size_t(up.stride(0));
        Matrix h{hidden, ""}, w{weight, ""};
        h.data = w.data = nullptr;
        if (a[9] != Py_None) {
            const at::Tensor &t = tensor(a[9], "grad_hidden must be a 2-D CUDA tensor");
            h = Matrix(t, "grad_hidden must be a 2-D CUDA tensor with contiguous rows");
            like(t, hidden);
        }
        if (a[10] != Py_None) {
            const at::Tensor &t = tensor(a[10], "grad_weight must be a 2-D CUDA tensor");
            w = Matrix(t, "grad_weight must be a 2-D CUDA tensor with contiguous rows");
            like(t, weight);
        }
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(hidden.device().index());
        size_t need = 0;
        if (const int rc = rd_vocab_loss_grad_workspace(&v, a[9] != Py_None, a[10] != Py_None, &need)) return status(rc);
        const Workspace ws(a[6], need, hidden.device(), stream);
        const float *at_up = static_cast<const float *>(up.data_ptr());
        const int rc = without_gil([&] {
            return rd_vocab_loss_grad(&v, static_cast<const float *>(at_lse), at_up, up_stride, h.data, h.stride, w.data, w.stride, ws.data, ws.size, stream);
        });
        return rc != RD_OK ? status(rc) : Py_NewRef(Py_None);
    });
}

uint64_t bits(PyObject *o)
{
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == ~0ull && PyErr_Occurred()) throw PythonError();
    return v;
}
size_t count(PyObject *o)
{
    const int64_t v = whole(o);
    if (v < 0) wrong("first_row must not be negative");
    return size_t(v);
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v;
}

// The given tensor, or a new one; [rows, dim] of a type on a device.
at::Tensor matrix_or_new(PyObject *given, size_t rows, size_t dim, at::ScalarType type, c10::Device device, const char *what)
{
    if (given == Py_None) return empty({int64_t(rows), int64_t(dim)}, type, device);
    const at::Tensor &t = tensor(given, what);
    if (t.dim() != 2 || size_t(t.size(0)) != rows || size_t(t.size(1)) != dim || t.scalar_type() != type || t.device() != device) wrong(what);
    return t;
}
const at::Tensor &weight_vector(PyObject *o, size_t dim, c10::Device device)
{
    const at::Tensor &t = tensor(o, "weight must be a CUDA vector");
    vector(t, dim, device, "weight must be a contiguous CUDA vector with one value per column, on the operands' device");
    return t;
}
PyObject *wrap_or_none(const at::Tensor &t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }

// x, weight, residual, eps, out_dtype, drop, seed, offset, first_row, out, total
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&]() -> PyObject * {
        const at::Tensor &x = tensor(a[0], "x must be a 2-D CUDA tensor");
        const Matrix m(x, "x must be a 2-D CUDA tensor with contiguous rows");
        const c10::Device device = x.device();
        const c10::cuda::OptionalCUDAGuard guard(device);
        const at::Tensor &weight = weight_vector(a[1], m.dim, device);
        rd_norm_t v{};
        v.x = m.data;
        v.x_stride = m.stride;
        v.weight = weight.data_ptr();
        v.n = m.rows;
        v.dim = m.dim;
        v.dtype = v.sum_dtype = code(x);
        v.weight_dtype = code(weight);
        v.eps = real(a[3]);
        v.drop = real(a[5]);
        v.seed = bits(a[6]);
        v.offset = bits(a[7]);
        v.first_row = count(a[8]);
        at::ScalarType out_type = x.scalar_type(), sum_type = x.scalar_type();
        if (a[4] != Py_None) {
            if (!THPDtype_Check(a[4])) wrong("out_dtype must be x's dtype or torch.float8_e4m3fn");
            out_type = reinterpret_cast<THPDtype *>(a[4])->scalar_type;
            if (out_type != x.scalar_type() && out_type != at::kFloat8_e4m3fn) wrong("out_dtype must be x's dtype or torch.float8_e4m3fn");
        }
        if (a[2] != Py_None) {
            const at::Tensor &residual = tensor(a[2], "residual must be a 2-D CUDA tensor");
            const Matrix r(residual, "residual must be a 2-D CUDA tensor with contiguous rows");
            if (r.rows != m.rows || r.dim != m.dim || residual.device() != device) wrong("residual must be [n, dim] on x's device");
            v.residual = r.data;
            v.residual_stride = r.stride;
            v.sum_dtype = code(residual);
            sum_type = residual.scalar_type();
        } else if (a[10] != Py_None) {
            sum_type = tensor(a[10], "total must be a 2-D CUDA tensor").scalar_type();
            v.sum_dtype = code(tensor(a[10], ""));
        }
        const at::Tensor out = matrix_or_new(a[9], m.rows, m.dim, out_type, device, "out must be [n, dim] of out_dtype on x's device");
        at::Tensor total, rstd = empty({int64_t(m.rows)}, at::kFloat, device), scale;
        const Matrix o(out, "out must be a 2-D CUDA tensor with contiguous rows");
        Matrix s = o;
        s.data = nullptr;
        if (a[2] != Py_None || a[10] != Py_None || v.drop != 0.0f) {
            total = matrix_or_new(a[10], m.rows, m.dim, sum_type, device, "total must be [n, dim] of residual's dtype on x's device");
            s = Matrix(total, "total must be a 2-D CUDA tensor with contiguous rows");
        }
        if (out_type == at::kFloat8_e4m3fn) scale = empty({int64_t(m.rows)}, at::kFloat, device);
        float *at_scale = scale.defined() ? static_cast<float *>(scale.data_ptr()) : nullptr, *at_rstd = static_cast<float *>(rstd.data_ptr());
        const rd_dtype_t out_code = code(out);
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(device.index());
        const int rc = without_gil([&] { return rd_norm(&v, o.data, o.stride, out_code, at_scale, s.data, s.stride, at_rstd, stream); });
        if (rc != RD_OK) return status(rc);
        PyObject *r = PyTuple_New(4);
        if (!r) throw PythonError();
        PyTuple_SET_ITEM(r, 0, a[9] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[9]));
        PyTuple_SET_ITEM(r, 1, a[10] == Py_None ? wrap_or_none(total) : Py_NewRef(a[10]));
        PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(rstd));
        PyTuple_SET_ITEM(r, 3, wrap_or_none(scale));
        return r;
    });
}

// grad_out, total, weight, rstd, grad_total, want_residual, want_weight, drop, seed, offset, first_row, grad_x, grad_residual, grad_weight, workspace
PyObject *norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 15, [&]() -> PyObject * {
        const at::Tensor &up = tensor(a[0], "grad_out must be a 2-D CUDA tensor"), &total = tensor(a[1], "total must be a 2-D CUDA tensor");
        const Matrix g(up, "grad_out must be a 2-D CUDA tensor with contiguous rows"), t(total, "total must be a 2-D CUDA tensor with contiguous rows");
        const c10::Device device = up.device();
        const c10::cuda::OptionalCUDAGuard guard(device);
        if (t.rows != g.rows || t.dim != g.dim || total.device() != device) wrong("total must be [n, dim] on grad_out's device");
        const at::Tensor &weight = weight_vector(a[2], g.dim, device), &rstd = tensor(a[3], "rstd must be a CUDA vector");
        rd_norm_grad_t v{};
        v.grad_out = g.data;
        v.grad_out_stride = g.stride;
        v.sum = t.data;
        v.sum_stride = t.stride;
        v.rstd = static_cast<const float *>(vector(rstd, g.rows, device, "rstd must be a contiguous CUDA vector with one value per row, on the operands' device"));
        if (rstd.scalar_type() != at::kFloat) wrong("rstd must be float32");
        v.weight = weight.data_ptr();
        v.n = g.rows;
        v.dim = g.dim;
        v.dtype = code(up);
        v.sum_dtype = code(total);
        v.weight_dtype = code(weight);
        if (a[4] != Py_None) {
            const at::Tensor &more = tensor(a[4], "grad_total must be a 2-D CUDA tensor");
            const Matrix m(more, "grad_total must be a 2-D CUDA tensor with contiguous rows");
            if (m.rows != g.rows || m.dim != g.dim || more.scalar_type() != total.scalar_type() || more.device() != device) wrong("grad_total must be [n, dim] with total's dtype and device");
            v.grad_sum = m.data;
            v.grad_sum_stride = m.stride;
        }
        const bool want_residual = truth(a[5]) || a[12] != Py_None, want_weight = truth(a[6]) || a[13] != Py_None;
        v.drop = real(a[7]);
        v.seed = bits(a[8]);
        v.offset = bits(a[9]);
        v.first_row = count(a[10]);
        const at::Tensor gx = matrix_or_new(a[11], g.rows, g.dim, up.scalar_type(), device, "grad_x must be [n, dim] with grad_out's dtype and device");
        // without dropout, in one type, the two gradients are the same matrix
        const bool shared = want_residual && a[12] == Py_None && v.drop == 0.0f && total.scalar_type() == up.scalar_type();
        at::Tensor gr, gw;
        const Matrix x(gx, "grad_x must be a 2-D CUDA tensor with contiguous rows");
        Matrix r = x;
        r.data = nullptr;
        if (want_residual && !shared) {
            gr = matrix_or_new(a[12], g.rows, g.dim, total.scalar_type(), device, "grad_residual must be [n, dim] with total's dtype and device");
            r = Matrix(gr, "grad_residual must be a 2-D CUDA tensor with contiguous rows");
        }
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(device.index());
        void *at_weight = nullptr;
        size_t need = 0;
        if (want_weight) {
            if (a[13] == Py_None) gw = empty({int64_t(g.dim)}, weight.scalar_type(), device);
            else gw = tensor(a[13], "grad_weight must be a CUDA vector");
            at_weight = vector(gw, g.dim, device, "grad_weight must be a contiguous CUDA vector with one value per column, on the operands' device");
            if (gw.scalar_type() != weight.scalar_type()) wrong("grad_weight must have weight's dtype");
            if (const int rc = rd_norm_grad_workspace(v.n, v.dim, &need)) return status(rc);
        }
        const Workspace w(a[14], need, device, stream);
        const int rc = without_gil([&] { return rd_norm_grad(&v, x.data, x.stride, r.data, r.stride, at_weight, w.data, w.size, stream); });
        if (rc != RD_OK) return status(rc);
        PyObject *o = PyTuple_New(3);
        if (!o) throw PythonError();
        PyObject *first = a[11] == Py_None ? THPVariable_Wrap(gx) : Py_NewRef(a[11]);
        PyTuple_SET_ITEM(o, 0, first);
        PyTuple_SET_ITEM(o, 1, shared ? Py_NewRef(first) : a[12] == Py_None ? wrap_or_none(gr) : Py_NewRef(a[12]));
        PyTuple_SET_ITEM(o, 2, a[13] == Py_None ? wrap_or_none(gw) : Py_NewRef(a[13]));
        return o;
    });
}

// x, drop, seed, offset, first_row, out
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 6, [&]() -> PyObject * {
        const at::Tensor &x = tensor(a[0], "x must be a 2-D CUDA tensor");
        const Matrix m(x, "x must be a 2-D CUDA tensor with contiguous rows");
        const c10::cuda::OptionalCUDAGuard guard(x.device());
        const at::Tensor out = matrix_or_new(a[5], m.rows, m.dim, x.scalar_type(), x.device(), "out must be [n, dim] with x's dtype and device");
        const Matrix o(out, "out must be a 2-D CUDA tensor with contiguous rows");
        const rd_dtype_t dtype = code(x);
        const float drop = real(a[1]);
        const uint64_t seed = bits(a[2]), offset = bits(a[3]);
        const size_t first = count(a[4]);
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(x.device().index());
        const int rc = without_gil([&] { return rd_dropout(m.data, m.stride, m.rows, m.dim, dtype, drop, seed, offset, first, o.data, o.stride, stream); });
        if (rc != RD_OK) return status(rc);
        return a[5] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[5]);
    });
}

const float *scale_vector(PyObject *o, size_t n, c10::Device device, const char *what)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, what);
    if (t.scalar_type() != at::kFloat) wrong(what);
    return static_cast<const float *>(vector(t, n, device, what));
}

// x, gate_weight, up_weight; x_scale, gate_scale, up_scale from `scales` on (null: none); activation
rd_gated_t projections(const at::Tensor &x, const at::Tensor &gate, const at::Tensor &up, PyObject *const *scales, PyObject *activation)
{
    const Matrix m(x, "x must be a 2-D CUDA tensor with contiguous rows"), g(gate, "gate_weight must be a 2-D CUDA tensor with contiguous rows"),
        u(up, "up_weight must be a 2-D CUDA tensor with contiguous rows");
    if (g.dim != m.dim || u.dim != m.dim || u.rows != g.rows || gate.scalar_type() != x.scalar_type() || up.scalar_type() != x.scalar_type() || gate.device() != x.device() ||
        up.device() != x.device())
        wrong("gate_weight and up_weight must be [width, dim] with x's dtype and device");
    rd_gated_t v{};
    v.x = m.data;
    v.x_stride = m.stride;
    v.gate_weight = g.data;
    v.gate_weight_stride = g.stride;
    v.up_weight = u.data;
    v.up_weight_stride = u.stride;
    v.n = m.rows;
    v.dim = m.dim;
    v.width = g.rows;
    v.dtype = code(x);
    const int64_t act = whole(activation);
    v.activation = static_cast<rd_activation_t>(act == int32_t(act) ? int32_t(act) : -1);      // -1: refused by the call
    if (scales) {
        v.x_scale = scale_vector(scales[0], m.rows, x.device(), "x_scale must be a contiguous float32 CUDA vector with one value per row, on the operands' device");
        v.gate_scale = scale_vector(scales[1], g.rows, x.device(), "gate_scale must be a contiguous float32 CUDA vector with one value per weight row, on the operands' device");
        v.up_scale = scale_vector(scales[2], g.rows, x.device(), "up_scale must be a contiguous float32 CUDA vector with one value per weight row, on the operands' device");
    }
    return v;
}

// x, gate_weight, up_weight, activation, keep, x_scale, gate_scale, up_scale, out_dtype, out, gate, up, workspace
PyObject *gated(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 13, [&]() -> PyObject * {
        const at::Tensor &x = tensor(a[0], "x must be a 2-D CUDA tensor");
        const rd_gated_t v = projections(x, tensor(a[1], "gate_weight must be a 2-D CUDA tensor"), tensor(a[2], "up_weight must be a 2-D CUDA tensor"), a + 5, a[3]);
        const c10::Device device = x.device();
        const c10::cuda::OptionalCUDAGuard guard(device);
        at::ScalarType type = x.scalar_type() == at::kFloat8_e4m3fn ? at::kBFloat16 : x.scalar_type();
        if (a[8] != Py_None) {
            if (!THPDtype_Check(a[8])) wrong("out_dtype must be a torch.dtype");
            type = reinterpret_cast<THPDtype *>(a[8])->scalar_type;
        }
        const bool keep = truth(a[4]);
        const char *const names[3] = {"out must be [n, width] of out_dtype on x's device", "gate must be [n, width] of out_dtype on x's device", "up must be [n, width] of out_dtype on x's device"};
        at::Tensor t[3];
        void *data[3] = {};
        size_t stride[3] = {};
        for (int k = 0; k < 3; k++) {
            if (k > 0 && !keep && a[9 + k] == Py_None) continue;
            t[k] = matrix_or_new(a[9 + k], v.n, v.width, type, device, names[k]);
            const Matrix m(t[k], names[k]);
            data[k] = m.data;
            stride[k] = m.stride;
        }
        const rd_dtype_t out_type = code(t[0]);
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(device.index());
        size_t need = 0;
        if (const int rc = rd_gated_workspace(&v, &need)) return status(rc);
        const Workspace w(a[12], need, device, stream);
        const int rc = without_gil([&] { return rd_gated(&v, data[0], stride[0], out_type, data[1], stride[1], data[2], stride[2], w.data, w.size, stream); });
        if (rc != RD_OK) return status(rc);
        PyObject *r = PyTuple_New(3);
        if (!r) throw PythonError();
        for (int k = 0; k < 3; k++) PyTuple_SET_ITEM(r, k, a[9 + k] == Py_None ? wrap_or_none(t[k]) : Py_NewRef(a[9 + k]));
        return r;
    });
}

// grad_out, x, gate_weight, up_weight, gate, up, activation, want_x, want_weights, grad_x, grad_gate_weight, grad_up_weight, workspace
PyObject *gated_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(n_args, 13, [&]() -> PyObject * {
        const at::Tensor &x = tensor(a[1], "x must be a 2-D CUDA tensor"), &gate_weight = tensor(a[2], "gate_weight must be a 2-D CUDA tensor");
        const at::Tensor &up_weight = tensor(a[3], "up_weight must be a 2-D CUDA tensor");
        const rd_gated_t v = projections(x, gate_weight, up_weight, nullptr, a[6]);
        const c10::Device device = x.device();
        const c10::cuda::OptionalCUDAGuard guard(device);
        const char *const names[3] = {"grad_out must be [n, width] with x's dtype and device", "gate must be [n, width] with x's dtype and device", "up must be [n, width] with x's dtype and device"};
        const void *in[3];
        size_t in_stride[3];
        PyObject *const given[3] = {a[0], a[4], a[5]};
        for (int k = 0; k < 3; k++) {
            const at::Tensor &t = tensor(given[k], names[k]);
            const Matrix m(t, names[k]);
            if (m.rows != v.n || m.dim != v.width || t.scalar_type() != x.scalar_type() || t.device() != device) wrong(names[k]);
            in[k] = m.data;
            in_stride[k] = m.stride;
        }
        const bool wanted[3] = {truth(a[7]), truth(a[8]), truth(a[8])};
        const char *const outs[3] = {"grad_x must be a 2-D CUDA tensor like x, with contiguous rows", "grad_gate_weight must be a 2-D CUDA tensor like gate_weight, with contiguous rows",
                                     "grad_up_weight must be a 2-D CUDA tensor like up_weight, with contiguous rows"};
        at::Tensor t[3];
        void *out[3] = {};
        size_t out_stride[3] = {};
        for (int k = 0; k < 3; k++) {
            if (!wanted[k] && a[9 + k] == Py_None) continue;
            t[k] = matrix_or_new(a[9 + k], k ? v.width : v.n, v.dim, x.scalar_type(), device, outs[k]);
            const Matrix m(t[k], outs[k]);
            out[k] = m.data;
            out_stride[k] = m.stride;
        }
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(device.index());
        size_t need = 0;
        if (const int rc = rd_gated_grad_workspace(&v, out[0] != nullptr, &need)) return status(rc);
        const Workspace w(a[12], need, device, stream);
        const int rc = without_gil([&] {
            return rd_gated_grad(&v, in[0], in_stride[0], in[1], in_stride[1], in[2], in_stride[2], out[0], out_stride[0], out[1], out_stride[1], out[2], out_stride[2], w.data, w.size, stream);
        });
        if (rc != RD_OK) return status(rc);
        PyObject *r = PyTuple_New(3);
        if (!r) throw PythonError();
        for (int k = 0; k < 3; k++) PyTuple_SET_ITEM(r, k, a[9 + k] == Py_None ? wrap_or_none(t[k]) : Py_NewRef(a[9 + k]));
        return r;
    });
}

PyMethodDef methods[] = {
    {"embed", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(embed)), METH_FASTCALL, nullptr},
    {"embed_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(embed_grad)), METH_FASTCALL, nullptr},
    {"vocab_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(vocab_loss)), METH_FASTCALL, nullptr},
    {"vocab_loss_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(vocab_loss_grad)), METH_FASTCALL, nullptr},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(norm)), METH_FASTCALL, nullptr},
    {"norm_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(norm_grad)), METH_FASTCALL, nullptr},
    {"dropout", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(dropout)), METH_FASTCALL, nullptr},
    {"gated", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gated)), METH_FASTCALL, nullptr},
    {"gated_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gated_grad)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rd_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rd_torch() { return PyModule_Create(&module); }
