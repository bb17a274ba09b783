// Python entries of the operators beside the sparse product on torch tensors: the look at the tensors, the outputs'
// and the workspace's allocation, the stream and the call of the library in one native function each, as a call in a
// decoding loop is over in a few us.
//
// PyTorch is used for device memory and streams only, as everywhere in this package.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/Context.h>
#include <ATen/EmptyTensor.h>
#include <ATen/hip/impl/HIPCachingAllocatorMasqueradingAsCUDA.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include <exception>

#include "../../../include/spmm_layers.h"

namespace {

struct others_run {
    PyThreadState *state = PyEval_SaveThread();
    ~others_run() { PyEval_RestoreThread(state); }
};

// A Python error that is set already.
struct raised {};

[[noreturn]] void refuse(PyObject *type, const char *what)
{
    PyErr_SetString(type, what);
    throw raised();
}

int32_t type_of(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return SPMM_F32;
    case at::kHalf: return SPMM_F16;
    case at::kBFloat16: return SPMM_BF16;
    case at::kChar: return SPMM_I8;
    default: return -1;
    }
}

// The tensor behind an argument, or none for None.
const at::Tensor *tensor_of(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a torch tensor", name);
        throw raised();
    }
    return &THPVariable_Unpack(o);
}

// torch keeps the imaginary part of a conjugate as memory of the other sign and a mark.
void unmarked(const at::Tensor &t, const char *name)
{
    if (!t.is_neg()) return;
    PyErr_Format(PyExc_ValueError, "%s is a view whose negation is still to be made (resolve_neg() makes it)", name);
    throw raised();
}

// A 2-D device tensor of the given types (a mask over SPMM_*) as the library sees it.
spmm_tensor_t seen(const at::Tensor &t, const char *name, unsigned types)
{
    const int32_t type = t.is_cuda() && t.layout() == at::kStrided && t.dim() == 2 ? type_of(t.scalar_type()) : -1;
    if (type < 0 || !(types >> type & 1)) {
        PyErr_Format(PyExc_ValueError, "%s must be a 2-D device tensor (features, tokens) of type %s", name,
                     types == 15u ? "float32, float16, bfloat16 or int8" : types == 8u ? "int8" : "float32, float16 or bfloat16");
        throw raised();
    }
    const int64_t rows = t.size(0), cols = t.size(1), s0 = t.stride(0), s1 = t.stride(1);
    if (rows > 0 && cols > 0 && !((s0 == 1 || rows == 1) && (cols == 1 || s1 >= rows)) && !((s1 == 1 || cols == 1) && (rows == 1 || s0 >= cols))) {
        PyErr_Format(PyExc_ValueError, "%s must have a stride of 1 along its features or its tokens, and no two elements in one place", name);
        throw raised();
    }
    unmarked(t, name);
    return {t.data_ptr(), s0, s1, type};
}

void sized(const at::Tensor &t, const char *name, int64_t rows, int64_t cols, const at::Tensor &beside)
{
    if (t.size(0) != rows || t.size(1) != cols) {
        PyErr_Format(PyExc_ValueError, "%s has shape (%lld, %lld), not (%lld, %lld)", name, (long long)t.size(0), (long long)t.size(1), (long long)rows, (long long)cols);
        throw raised();
    }
    if (t.device() != beside.device()) {
        PyErr_Format(PyExc_ValueError, "%s is on another device", name);
        throw raised();
    }
}

// A vector of `n` elements without gaps beside `beside`.
void vector_of(const at::Tensor &t, const char *name, int64_t n, bool floats_only, const at::Tensor &beside)
{
    const int32_t type = type_of(t.scalar_type());
    if (!(t.is_cuda() && t.dim() == 1 && t.size(0) == n && (n <= 1 || t.stride(0) == 1) && t.device() == beside.device() &&
          (floats_only ? type == SPMM_F32 : type >= SPMM_F32 && type <= SPMM_BF16))) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous %s device tensor of %lld elements", name, floats_only ? "float32" : "float32, float16 or bfloat16", (long long)n);
        throw raised();
    }
    unmarked(t, name);
}

// The device has to be the current one, as plans and streams are bound to theirs.
void on_current_device(const at::Tensor &t)
{
    if (c10::hip::current_device() != t.device().index()) refuse(PyExc_ValueError, "the tensors' device is not the current one");
}

// By token: a row of memory is a token.
bool by_token(const at::Tensor &t) { return t.stride(1) != 1 && t.stride(0) == 1; }

// Allocations of a call.  On its way through the dispatcher at::empty takes 0.3 us of a small call's 3 to 4, and a norm makes three tensors.  Where nothing may
// want to see or change those calls (a dispatch mode, a functional transform, inference mode, a profiler, the fill of deterministic mode) they are
// made from the same allocator directly.
struct allocations {
    const at::Tensor &beside;
    bool plain;
    explicit allocations(const at::Tensor &t) : beside(t)
    {
        const c10::impl::LocalDispatchKeySet local = c10::impl::tls_local_dispatch_key_set();
        plain = local.included_ == c10::default_included_set && local.excluded_ == c10::default_excluded_set && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
                !at::hasCallbacks() && !at::globalContext().deterministicAlgorithms() && t.key_set().has(c10::DispatchKey::CUDA);
    }
    at::Tensor strided(at::IntArrayRef sizes, at::IntArrayRef strides, at::ScalarType type) const
    {
        if (!plain) return at::empty_strided(sizes, strides, at::TensorOptions().dtype(type).device(beside.device()));
        return at::Tensor(at::detail::empty_strided_generic(sizes, strides, c10::hip::HIPCachingAllocatorMasqueradingAsCUDA::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type));
    }
    // (rows, cols), a row or a column of it in a piece
    at::Tensor matrix(int64_t rows, int64_t cols, bool columns, at::ScalarType type) const
    {
        const int64_t sizes[2] = {rows, cols}, strides[2] = {columns ? 1 : cols, columns ? rows : 1};
        return strided(sizes, strides, type);
    }
    at::Tensor vector(int64_t n, at::ScalarType type) const
    {
        const int64_t one = 1;
        return strided(n, one, type);
    }
};

at::ScalarType dtype_of(PyObject *o, at::ScalarType otherwise, unsigned types)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) refuse(PyExc_TypeError, "dtype must be a torch.dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
    const int32_t type = type_of(t);
    if (type < 0 || !(types >> type & 1)) refuse(PyExc_ValueError, types == 15u ? "dtype must be float32, float16, bfloat16 or int8" : "dtype must be float32, float16 or bfloat16");
    return t;
}

void *stream_beside(const at::Tensor &t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

struct workspace {
    at::Tensor memory;
    void *data = nullptr;
    size_t bytes = 0;
    void take(size_t n, const allocations &from)
    {
        if (n == 0) return;
        memory = from.vector((int64_t)n, at::kByte);
        data = memory.data_ptr();
        bytes = n;
    }
};

PyObject *wrapped(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

// The named tuples of layers.py, which norm and gate answer with.
PyTypeObject *normed_type = nullptr, *gated_type = nullptr;

PyObject *answer_types(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs != 2 || !PyType_Check(args[0]) || !PyType_Check(args[1]) || !PyType_IsSubtype((PyTypeObject *)args[0], &PyTuple_Type) ||
        !PyType_IsSubtype((PyTypeObject *)args[1], &PyTuple_Type)) {
        PyErr_SetString(PyExc_TypeError, "answer_types(Normed, Gated)");
        return nullptr;
    }
    Py_INCREF(args[0]);
    Py_INCREF(args[1]);
    normed_type = (PyTypeObject *)args[0], gated_type = (PyTypeObject *)args[1];
    Py_RETURN_NONE;
}

// A tuple of the given subclass; takes over the references of `fields`.
template <int N> PyObject *answer(PyTypeObject *type, PyObject *const (&fields)[N])
{
    PyObject *t = type ? type->tp_alloc(type, N) : PyTuple_New(N);
    for (int i = 0; i < N; ++i) {
        if (t && fields[i]) PyTuple_SET_ITEM(t, i, fields[i]);
        else Py_XDECREF(fields[i]);
    }
    if (!PyErr_Occurred()) return t;
    Py_XDECREF(t);
    return nullptr;
}

template <typename F> PyObject *guarded(F &&f)
{
    try {
        return f();
    } catch (const raised &) {
        return nullptr;
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

PyObject *wrong_count(const char *what)
{
    PyErr_SetString(PyExc_TypeError, what);
    return nullptr;
}

constexpr unsigned FLOATS = 7u, ANY = 15u;

// quant_execute(plan address, M, K, B, C or None, B's scales or None, dtype or None) -> C, or the status code as int
PyObject *quant_execute(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs != 7) return wrong_count("quant_execute(plan, M, K, B, C, scales, dtype)");
    const spmm_quant_t *plan = static_cast<const spmm_quant_t *>(PyLong_AsVoidPtr(args[0]));
    const int64_t M = PyLong_AsLongLong(args[1]), K = PyLong_AsLongLong(args[2]);
    if (PyErr_Occurred()) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *B = tensor_of(args[3], "B"), *given = tensor_of(args[4], "C"), *scales = tensor_of(args[5], "scales");
        if (!B) refuse(PyExc_TypeError, "B must be a torch tensor");
        const spmm_tensor_t b = seen(*B, "B", ANY);
        const int64_t N = B->size(1);
        sized(*B, "B", K, N, *B);
        if (N > INT32_MAX) refuse(PyExc_ValueError, "B has more columns than the library's 31-bit column count");
        on_current_device(*B);
        if (b.type == SPMM_I8) {
            if (!scales) refuse(PyExc_ValueError, "B in codes comes with its tokens' scales");
            vector_of(*scales, "scales", N, true, *B);
            if (K > 1 && N > 0 && B->stride(0) != 1) refuse(PyExc_ValueError, "B in codes must hold one token a row of memory (stride 1 along its features)");
        } else if (scales) {
            refuse(PyExc_ValueError, "scales belong to a B in codes");
        }
        at::Tensor C;
        if (given) {
            seen(*given, "C", FLOATS);
            sized(*given, "C", M, N, *B);
            if (args[6] != Py_None && dtype_of(args[6], at::kFloat, FLOATS) != given->scalar_type()) refuse(PyExc_ValueError, "dtype is not C's");
            C = *given;
        }
        const at::ScalarType type = dtype_of(args[6], b.type == SPMM_I8 ? at::kFloat : B->scalar_type(), FLOATS);
        spmm_status_t st;
        {
            others_run free_to_run;
            const allocations from(*B);
            if (!given) C = from.matrix(M, N, by_token(*B), type);
            const spmm_tensor_t c = {C.data_ptr(), C.stride(0), C.stride(1), type_of(C.scalar_type())};
            size_t bytes = 0;
            workspace room;
            st = spmm_quant_workspace(plan, &b, N, &bytes);
            if (st == SPMM_OK) {
                room.take(bytes, from);
                st = spmm_quant_execute(plan, &b, scales ? static_cast<const float *>(scales->data_ptr()) : nullptr, N, &c, room.data, room.bytes, stream_beside(*B));
            }
        }
        if (st != SPMM_OK) return PyLong_FromLong((long)st);
        if (!given) return THPVariable_Wrap(std::move(C));
        Py_INCREF(args[4]);
        return args[4];
    });
}

// What norm and gate share: the outputs.
struct outputs {
    at::Tensor out, scales;
    void look(PyObject *out_arg, PyObject *scales_arg, PyObject *dtype_arg, const at::Tensor &x, at::ScalarType *type)
    {
        const at::Tensor *o = tensor_of(out_arg, "out"), *s = tensor_of(scales_arg, "scales");
        if (o) {
            seen(*o, "out", ANY);
            sized(*o, "out", x.size(0), x.size(1), x);
            if (dtype_arg != Py_None && dtype_of(dtype_arg, at::kFloat, ANY) != o->scalar_type()) refuse(PyExc_ValueError, "dtype is not out's");
            out = *o;
        }
        *type = o ? o->scalar_type() : dtype_of(dtype_arg, x.scalar_type(), ANY);
        if (s) {
            if (*type != at::kChar) refuse(PyExc_ValueError, "scales belong to an output in codes");
            vector_of(*s, "scales", x.size(1), true, x);
            scales = *s;
        }
    }
    void make(const at::Tensor &x, at::ScalarType type, const allocations &from)
    {
        if (!out.defined()) out = from.matrix(x.size(0), x.size(1), type == at::kChar || by_token(x), type);
        if (type == at::kChar && !scales.defined()) scales = from.vector(x.size(1), at::kFloat);
    }
};

void in_range(const at::Tensor &x)
{
    if (x.size(0) < 1 || x.size(1) < 1 || x.size(0) > INT32_MAX || x.size(1) > INT32_MAX) refuse(PyExc_ValueError, "features and tokens must be 1 .. 2^31 - 1");
}

spmm_tensor_t as_seen(const at::Tensor &t)
{
    if (!t.defined()) return {nullptr, 0, 0, SPMM_F32};
    return {t.data_ptr(), t.stride(0), t.stride(1), type_of(t.scalar_type())};
}

// norm(x, weight, eps, residual, total, wants total, out, scales, dtype) -> (out, total, scales), or the status code
PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs != 9) return wrong_count("norm(x, weight, eps, residual, total, wants_total, out, scales, dtype)");
    const double eps = PyFloat_AsDouble(args[2]);
    const int wants = PyObject_IsTrue(args[5]);
    if (PyErr_Occurred()) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *x = tensor_of(args[0], "x"), *w = tensor_of(args[1], "weight"), *r = tensor_of(args[3], "residual"), *t = tensor_of(args[4], "total");
        if (!x || !w) refuse(PyExc_TypeError, "x and weight must be torch tensors");
        spmm_norm_t a = {};
        a.x = seen(*x, "x", FLOATS);
        in_range(*x);
        on_current_device(*x);
        vector_of(*w, "weight", x->size(0), false, *x);
        at::Tensor total;
        if (r) {
            a.residual = seen(*r, "residual", 1u << a.x.type);
            sized(*r, "residual", x->size(0), x->size(1), *x);
        }
        if (t) {
            seen(*t, "total", 1u << a.x.type);
            sized(*t, "total", x->size(0), x->size(1), *x);
            total = *t;
        }
        outputs o;
        at::ScalarType type;
        o.look(args[6], args[7], args[8], *x, &type);
        spmm_status_t st;
        {
            others_run free_to_run;
            const allocations from(*x);
            o.make(*x, type, from);
            if (wants && !t) total = from.matrix(x->size(0), x->size(1), by_token(*x), x->scalar_type());
            a.total = as_seen(total);
            a.out = as_seen(o.out);
            a.scales = o.scales.defined() ? static_cast<float *>(o.scales.data_ptr()) : nullptr;
            a.weight = w->data_ptr();
            a.weight_type = type_of(w->scalar_type());
            a.eps = (float)eps;
            size_t bytes = 0;
            workspace room;
            st = spmm_norm_workspace(x->size(0), x->size(1), &a, &bytes);
            if (st == SPMM_OK) {
                room.take(bytes, from);
                st = spmm_norm(x->size(0), x->size(1), &a, room.data, room.bytes, stream_beside(*x));
            }
        }
        if (st != SPMM_OK) return PyLong_FromLong((long)st);
        return answer<3>(normed_type, {wrapped(o.out), wrapped(total), wrapped(o.scales)});
    });
}

// gate(a, b, act, out, scales, dtype) -> (out, scales), or the status code
PyObject *gate(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs != 6) return wrong_count("gate(a, b, act, out, scales, dtype)");
    const long act = PyLong_AsLong(args[2]);
    if (PyErr_Occurred()) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *x = tensor_of(args[0], "a"), *b = tensor_of(args[1], "b");
        if (!x) refuse(PyExc_TypeError, "a must be a torch tensor");
        spmm_gate_t g = {};
        g.a = seen(*x, "a", FLOATS);
        in_range(*x);
        on_current_device(*x);
        if (b) {
            g.b = seen(*b, "b", 1u << g.a.type);
            sized(*b, "b", x->size(0), x->size(1), *x);
        }
        outputs o;
        at::ScalarType type;
        o.look(args[3], args[4], args[5], *x, &type);
        spmm_status_t st;
        {
            others_run free_to_run;
            const allocations from(*x);
            o.make(*x, type, from);
            g.out = as_seen(o.out);
            g.scales = o.scales.defined() ? static_cast<float *>(o.scales.data_ptr()) : nullptr;
            g.act = (int32_t)act;
            size_t bytes = 0;
            workspace room;
            st = spmm_gate_workspace(x->size(0), x->size(1), &g, &bytes);
            if (st == SPMM_OK) {
                room.take(bytes, from);
                st = spmm_gate(x->size(0), x->size(1), &g, room.data, room.bytes, stream_beside(*x));
            }
        }
        if (st != SPMM_OK) return PyLong_FromLong((long)st);
        return answer<2>(gated_type, {wrapped(o.out), wrapped(o.scales)});
    });
}

PyMethodDef methods[] = {
    {"quant_execute", (PyCFunction)(void (*)(void))quant_execute, METH_FASTCALL, "spmm_quant_execute on torch tensors; returns C, or a status code"},
    {"norm", (PyCFunction)(void (*)(void))norm, METH_FASTCALL, "spmm_norm on torch tensors; returns (out, total, scales), or a status code"},
    {"gate", (PyCFunction)(void (*)(void))gate, METH_FASTCALL, "spmm_gate on torch tensors; returns (out, scales), or a status code"},
    {"answer_types", (PyCFunction)(void (*)(void))answer_types, METH_FASTCALL, "answer_types(Normed, Gated): the tuples that norm and gate answer with"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_spmm_layers", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__spmm_layers(void) { return PyModule_Create(&module_def); }
