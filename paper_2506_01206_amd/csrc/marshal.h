// What the parts of the binding's marshalling module (marshal.cpp, marshal_delta.cpp, marshal_sample.cpp) share: checks of tensors, outputs and
// scratch allocated for the caller, the call into the C ABI and its errors.
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "../../include/mamba_hip.h"

namespace {

// a Python exception is already set
struct PyFailed {};

PyObject *mamba_error = nullptr;      // binding.MambaError(function name, status)
PyObject *out_of_memory = nullptr;    // torch.OutOfMemoryError

typedef std::initializer_list<int64_t> Shape;

[[noreturn]] void fail(PyObject *type, const char *format, const char *name)
{
    PyErr_Format(type, format, name);
    throw PyFailed();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}

// sizes of a tensor that has to have `rank` dimensions, or at least as many
at::IntArrayRef sizes(PyObject *o, const char *name, size_t rank, bool or_more = false)
{
    const at::IntArrayRef s = tensor(o, name).sizes();
    if (s.size() < rank || (s.size() > rank && !or_more)) {
        PyErr_Format(PyExc_ValueError, "%s must have %s%zu dimensions, got %zu", name, or_more ? "at least " : "", rank, s.size());
        throw PyFailed();
    }
    return s;
}

void *pointer(const at::Tensor &t) { return t.numel() > 0 ? t.data_ptr() : nullptr; }

void placed(const at::Tensor &t, const char *name)
{
    if (!t.is_cuda()) fail(PyExc_ValueError, "%s must live on the GPU", name);
    if (!t.is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
}

PyObject *dtype_object(at::ScalarType type) { return reinterpret_cast<PyObject *>(torch::getTHPDtype(type)); }   // borrowed

void typed(const at::Tensor &t, at::ScalarType type, const char *name)
{
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must be %S, got %S", name, dtype_object(type), dtype_object(t.scalar_type()));
        throw PyFailed();
    }
}

std::string text(at::IntArrayRef shape)   // as Python writes a tuple
{
    std::string s = "(";
    for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
    return s + (shape.size() == 1 ? ",)" : ")");
}

void shaped(const at::Tensor &t, Shape shape, const char *name)
{
    const at::IntArrayRef s = t.sizes();
    if (s == at::IntArrayRef(shape)) return;
    PyErr_Format(PyExc_ValueError, "%s must have shape %s, got %s", name, text(shape).c_str(), text(s).c_str());
    throw PyFailed();
}

// device pointer of a contiguous GPU tensor (None: NULL)
void *ptr(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    placed(t, name);
    return pointer(t);
}
[[maybe_unused]] void *ptr(PyObject *o, at::ScalarType type, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    placed(t, name);
    typed(t, type, name);
    return pointer(t);
}
void *ptr(PyObject *o, at::ScalarType type, Shape shape, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    placed(t, name);
    typed(t, type, name);
    shaped(t, shape, name);
    return pointer(t);
}
float *fptr(PyObject *o, Shape shape, const char *name) { return static_cast<float *>(ptr(o, at::kFloat, shape, name)); }

// all of these are tensors or None, and the checks before have seen to it that the tensors are the GPU's
[[maybe_unused]] void on_current_device(std::initializer_list<PyObject *> objects)
{
    const int current = c10::hip::current_device();
    for (PyObject *o : objects)
        if (o != Py_None && tensor(o, "tensor").get_device() != current) {
            PyErr_Format(PyExc_ValueError, "all tensors must live on the current device (%d), one lives on %d", current,
                         (int)tensor(o, "tensor").get_device());
            throw PyFailed();
        }
}

int io_code(const at::Tensor &t)
{
    if (t.scalar_type() == at::kFloat) return MAMBA_F32;
    if (t.scalar_type() == at::kBFloat16) return MAMBA_BF16;
    PyErr_Format(PyExc_TypeError, "I/O tensors must be float32 or bfloat16, got %S", dtype_object(t.scalar_type()));
    throw PyFailed();
}

int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyFailed();
    return v;
}
int flag(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PyFailed();
    return v;
}

// stream: the raw stream as an int, None for the current one
void *stream_of(PyObject *o)
{
    if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
    return reinterpret_cast<void *>(integer(o));
}

// An output: the caller's tensor, or one allocated here (then `owned` keeps it, and the result refers to it).
struct Out {
    PyObject *object;                 // borrowed (caller's tensor or None) until made
    PyObject *owned = nullptr;
    explicit Out(PyObject *o) : object(o) {}
    Out(const Out &) = delete;
    ~Out() { Py_XDECREF(owned); }
    void make(const at::Tensor &like, at::IntArrayRef shape, at::ScalarType type)
    {
        owned = THPVariable_Wrap(at::empty(shape, like.options().dtype(type)));
        if (!owned) throw PyFailed();
        object = owned;
    }
    void make(const at::Tensor &like, Shape shape, at::ScalarType type) { make(like, at::IntArrayRef(shape), type); }
    void unless_given(const at::Tensor &like, at::IntArrayRef shape, at::ScalarType type)
    {
        if (object == Py_None) make(like, shape, type);
    }
    void unless_given(const at::Tensor &like, Shape shape, at::ScalarType type) { unless_given(like, at::IntArrayRef(shape), type); }
};

// Scratch of one call.  The caching allocator may hand the block to later work on the current stream as soon as the
// call returns, so a call on another stream (`stream` given) is marshalled with the workspace binding.py allocates.
struct Workspace {
    at::Tensor own;
    void *data = nullptr;
    size_t bytes = 0;
    Workspace(PyObject *given, size_t need, const at::Tensor &like)
    {
        if (given != Py_None) {
            const at::Tensor &t = tensor(given, "workspace");
            data = ptr(given, "workspace");
            bytes = t.numel() * t.element_size();
        } else if (need > 0) {
            own = at::empty({(int64_t)(need < 16 ? 16 : need)}, like.options().dtype(at::kByte));
            data = own.data_ptr();
            bytes = (size_t)own.numel();
        }
    }
};

// Calls a function of the C ABI, the interpreter lock released meanwhile (a launch can block on a full queue), and
// raises MambaError for a status that is not zero.  A class, to be used with braces: only there are the arguments, which do
// the checks, formed in the order in which they are written (the current stream last, when all tensors are known to be the GPU's).
template <typename F, typename... A> struct Call {
    Call(const char *function, F f, A... args)
    {
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = f(args...);
        Py_END_ALLOW_THREADS
        if (status == 0) return;
        PyObject *e = PyObject_CallFunction(mamba_error, "si", function, status);
        if (e) {
            PyErr_SetObject(mamba_error, e);
            Py_DECREF(e);
        }
        throw PyFailed();
    }
};

PyObject *result(PyObject *const *first, PyObject *const *last)
{
    PyObject *t = PyTuple_New((Py_ssize_t)(last - first));
    if (!t) throw PyFailed();
    for (Py_ssize_t i = 0; i < last - first; ++i) {
        Py_INCREF(first[i]);
        PyTuple_SET_ITEM(t, i, first[i]);
    }
    return t;
}
PyObject *result(std::initializer_list<PyObject *> items) { return result(items.begin(), items.end()); }

typedef PyObject *const *Args;

// argument count, PyFailed and C++ exceptions (an allocation that fails) in one place
template <PyObject *(*F)(Args), int COUNT> PyObject *entry(PyObject *, Args args, Py_ssize_t n)
{
    if (n != COUNT) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", COUNT, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const PyFailed &) {
        return nullptr;
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(out_of_memory, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// bind(MambaError, torch.OutOfMemoryError, address, address, ...): the C functions in the order of the members of Api
template <typename Api, Api *api> PyObject *bind_to(Args args, Py_ssize_t n)
{
    constexpr Py_ssize_t count = sizeof(Api) / sizeof(void *);
    if (n != 2 + count) {
        PyErr_SetString(PyExc_TypeError, "bind: two exception classes and one address per function");
        return nullptr;
    }
    void **slot = reinterpret_cast<void **>(api);
    for (Py_ssize_t i = 0; i < count; ++i) {
        slot[i] = PyLong_AsVoidPtr(args[2 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(args[0]);
    Py_XSETREF(mamba_error, args[0]);
    Py_INCREF(args[1]);
    Py_XSETREF(out_of_memory, args[1]);
    Py_RETURN_NONE;
}

#define MAMBA_ENTRY(F, COUNT) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, COUNT>)), METH_FASTCALL, nullptr}

}  // namespace
