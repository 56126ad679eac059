// The operators along time from Python: what a call depends on of its tensors as one key, and the call itself.
//
// One token's kernels run for 3 us.  Types, shapes, strides and addresses of some ten tensors read through Python and passed through ctypes took longer
// than that (norm of one token of 8 + 8 heads of 64: 7.8 us a call, read here 4.9; one step of 8 heads of 64: 7.7 and 5.1).  Nothing is decided here: checks are made by the
// binding and by the library, and nothing is kept between calls but the library's entry points.
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/tfno.h"

namespace {

constexpr int MOST = 32, MOST_AXES = 8;       // tensors of a call, and axes of one

struct Library {
    decltype(&tfno_head_norm_rope) norm;
    decltype(&tfno_head_norm_rope_backward) norm_backward;
    decltype(&tfno_gated_delta_rule) rule;
    decltype(&tfno_gated_delta_rule_backward) rule_backward;
    decltype(&tfno_gated_delta_rule_step) step;
} library;

// Numbers of any size in few bytes: seven bits in each, the last one below 128.
unsigned char *put(unsigned char *at, int64_t value)
{
    uint64_t left = (uint64_t)value << 1 ^ (uint64_t)(value >> 63);
    for (; left >= 128; left >>= 7) *at++ = (unsigned char)(left | 128);
    *at++ = (unsigned char)left;
    return at;
}

PyObject *key(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    unsigned char bytes[MOST * (3 + 2 * MOST_AXES) * 10], *at = bytes;
    if (count > MOST) return PyErr_Format(PyExc_ValueError, "more than %d tensors", MOST);
    try {
        for (Py_ssize_t i = 0; i < count; ++i) {
            if (args[i] == Py_None) {
                at = put(at, -1);
                continue;
            }
            if (!THPVariable_Check(args[i])) return PyErr_Format(PyExc_TypeError, "a tensor is expected, not %.100s", Py_TYPE(args[i])->tp_name);
            const at::Tensor &t = THPVariable_Unpack(args[i]);
            if (t.layout() != at::kStrided || t.dim() > MOST_AXES) return PyErr_Format(PyExc_ValueError, "tensors must be dense, with at most %d axes", MOST_AXES);
            if (t.is_neg() || t.is_conj()) return PyErr_Format(PyExc_ValueError, "a tensor's memory must hold its values: resolve_neg() and resolve_conj() first");
            at = put(at, t.dim());
            at = put(at, (int64_t)t.scalar_type());
            at = put(at, t.is_cuda() ? t.get_device() : -1);
            for (int64_t n : t.sizes()) at = put(at, n);
            for (int64_t n : t.strides()) at = put(at, n);
        }
    } catch (const std::exception &e) {
        return PyErr_Format(PyExc_RuntimeError, "%.300s", e.what());
    }
    return PyBytes_FromStringAndSize((const char *)bytes, at - bytes);
}

// An argument of an entry point: of a pointer a tensor, an address or None, of an int a number.  PyErr_Occurred() says whether it was one.
template <class A>
A argument(PyObject *x)
{
    if constexpr (std::is_pointer_v<A>) {
        if (x == Py_None) return nullptr;
        if (THPVariable_Check(x)) return (A)THPVariable_Unpack(x).data_ptr();
        return (A)PyLong_AsVoidPtr(x);
    } else {
        static_assert(std::is_same_v<A, int>);
        const long value = PyLong_AsLong(x);
        if ((int)value != value) PyErr_SetString(PyExc_OverflowError, "a number does not fit 32 bits");
        return (int)value;
    }
}

template <class... A, size_t... I>
PyObject *call(tfno_status (*entry)(A...), PyObject *const *args, Py_ssize_t count, std::index_sequence<I...>)
{
    if (!entry) return PyErr_Format(PyExc_RuntimeError, "the library is not open");
    if (count != (Py_ssize_t)sizeof...(A)) return PyErr_Format(PyExc_TypeError, "%d arguments are expected, not %d", (int)sizeof...(A), (int)count);
    tfno_status st;
    try {
        std::tuple<A...> a{argument<A>(args[I])...};
        if (PyErr_Occurred()) return nullptr;
        Py_BEGIN_ALLOW_THREADS
        st = entry(std::get<I>(a)...);
        Py_END_ALLOW_THREADS
    } catch (const std::exception &e) {       // a tensor without memory; the library's entry points throw nothing
        return PyErr_Format(PyExc_RuntimeError, "%.300s", e.what());
    }
    return PyLong_FromLong(st);
}

template <class... A>
PyObject *call(tfno_status (*entry)(A...), PyObject *const *args, Py_ssize_t count)
{
    return call(entry, args, count, std::index_sequence_for<A...>{});
}

PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.norm, args, count); }
PyObject *norm_backward(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.norm_backward, args, count); }
PyObject *rule(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.rule, args, count); }
PyObject *rule_backward(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.rule_backward, args, count); }
PyObject *step(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.step, args, count); }

PyObject *open_library(PyObject *, PyObject *path)
{
    const char *name = PyUnicode_AsUTF8(path);
    if (!name) return nullptr;
    void *handle = dlopen(name, RTLD_NOW | RTLD_LOCAL);
    if (!handle) return PyErr_Format(PyExc_RuntimeError, "%.300s", dlerror());
    Library found;
    const auto find = [&](auto &entry, const char *symbol) {
        entry = (std::remove_reference_t<decltype(entry)>)dlsym(handle, symbol);
        if (!entry) PyErr_Format(PyExc_RuntimeError, "%.200s has no %s", name, symbol);
        return entry != nullptr;
    };
    if (!find(found.norm, "tfno_head_norm_rope") || !find(found.norm_backward, "tfno_head_norm_rope_backward") ||
        !find(found.rule, "tfno_gated_delta_rule") || !find(found.rule_backward, "tfno_gated_delta_rule_backward") ||
        !find(found.step, "tfno_gated_delta_rule_step"))
        return nullptr;
    library = found;
    Py_RETURN_NONE;
}

PyCFunction fast(PyObject *(*f)(PyObject *, PyObject *const *, Py_ssize_t)) { return (PyCFunction)(void *)f; }

PyMethodDef methods[] = {
    {"open", open_library, METH_O, "Finds the entry points in the library of this path."},
    {"key", fast(key), METH_FASTCALL, "Types, devices, shapes and strides of tensors (or None) as bytes: equal for equal ones."},
    {"tfno_head_norm_rope", fast(norm), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_head_norm_rope_backward", fast(norm_backward), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_gated_delta_rule", fast(rule), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_gated_delta_rule_backward", fast(rule_backward), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_gated_delta_rule_step", fast(step), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
