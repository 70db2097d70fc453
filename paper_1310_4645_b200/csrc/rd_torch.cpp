// Marshalling of the vocabulary operators' tensors: the same checks and calls that ctypes would make, without the interpreter.
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
    default: break;
    }
    PyErr_SetString(PyExc_TypeError, "int32, float32, int64, float64, bfloat16 or float16 expected");
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

PyMethodDef methods[] = {
    {"embed", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(embed)), METH_FASTCALL, nullptr},
    {"embed_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(embed_grad)), METH_FASTCALL, nullptr},
    {"vocab_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(vocab_loss)), METH_FASTCALL, nullptr},
    {"vocab_loss_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(vocab_loss_grad)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rd_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rd_torch() { return PyModule_Create(&module); }
