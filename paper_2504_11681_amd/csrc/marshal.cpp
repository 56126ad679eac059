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
#include <vector>

#include "../../include/tfno.h"

namespace {

constexpr int MOST = 32, MOST_AXES = 8;       // tensors of a call, and axes of one

struct Library {
    decltype(&tfno_head_norm_rope) norm;
    decltype(&tfno_head_norm_rope_backward) norm_backward;
    decltype(&tfno_gated_delta_rule) rule;
    decltype(&tfno_gated_delta_rule_backward) rule_backward;
    decltype(&tfno_gated_delta_rule_step) step;
    decltype(&tfno_gated_recurrence) recurrence;
    decltype(&tfno_gated_recurrence_backward) recurrence_backward;
    decltype(&tfno_gated_recurrence_step) recurrence_step;
    decltype(&tfno_block_norm) block_norm;
    decltype(&tfno_block_norm_backward) block_norm_backward;
    decltype(&tfno_clip_grad_norm) clip;
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

PyObject *recurrence(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.recurrence, args, count); }
PyObject *recurrence_backward(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.recurrence_backward, args, count); }
PyObject *recurrence_step(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.recurrence_step, args, count); }
PyObject *block_norm(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.block_norm, args, count); }
PyObject *block_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t count) { return call(library.block_norm_backward, args, count); }

// Tensors of any number (None is skipped) as the entry point takes them, and its call: (tensors, limit, norm or None, device, stream).  Here are all checks of the tensors' types and
// layouts: through Python they took longer than the kernels of a small model.
PyObject *clip(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    if (!library.clip) return PyErr_Format(PyExc_RuntimeError, "the library is not open");
    if (count != 5) return PyErr_Format(PyExc_TypeError, "5 arguments are expected, not %d", (int)count);
    const double limit = PyFloat_AsDouble(args[1]);
    const long device = PyLong_AsLong(args[3]);
    void *stream = PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) return nullptr;
    PyObject *list = PySequence_Fast(args[0], "the tensors must be a sequence");
    if (!list) return nullptr;
    PyObject *result = nullptr;
    try {
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
        PyObject **items = PySequence_Fast_ITEMS(list);
        std::vector<tfno_tensor> tensors((size_t)n);
        const char *wrong = nullptr;
        size_t there = 0;
        for (Py_ssize_t i = 0; i < n && !wrong; ++i) {
            if (items[i] == Py_None) continue;         // of a parameter without a gradient
            if (!THPVariable_Check(items[i])) {
                wrong = "gradients must be tensors";
                break;
            }
            const at::Tensor &t = THPVariable_Unpack(items[i]);
            const at::ScalarType type = t.scalar_type();
            if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) wrong = "gradients must be dense tensors on one device";
            else if (type != at::kFloat && type != at::kBFloat16 && type != at::kComplexFloat) wrong = "gradients must be float32, bfloat16 or complex64";
            else if (!t.is_non_overlapping_and_dense()) wrong = "gradients must fill their memory, in whatever order of axes";
            else tensors[there++] = {t.numel() ? t.data_ptr() : nullptr, (long long)t.numel() * (type == at::kComplexFloat ? 2 : 1), type == at::kBFloat16 ? TFNO_BF16 : TFNO_F32};
        }
        float *norm = nullptr;
        if (!wrong && args[2] != Py_None) {
            const bool tensor = THPVariable_Check(args[2]);
            if (!tensor || THPVariable_Unpack(args[2]).scalar_type() != at::kFloat || THPVariable_Unpack(args[2]).numel() != 1 ||
                !THPVariable_Unpack(args[2]).is_cuda() || THPVariable_Unpack(args[2]).get_device() != device)
                wrong = "norm must be one float32 on the device of the gradients";
            else norm = (float *)THPVariable_Unpack(args[2]).data_ptr();
        }
        if (wrong) {
            PyErr_SetString(PyExc_TypeError, wrong);
        } else {
            tfno_status st;
            Py_BEGIN_ALLOW_THREADS
            st = library.clip(tensors.data(), (int)there, limit, norm, stream);
            Py_END_ALLOW_THREADS
            result = PyLong_FromLong(st);
        }
    } catch (const std::exception &e) {       // a tensor without memory, or none on the host
        PyErr_Format(PyExc_RuntimeError, "%.300s", e.what());
    }
    Py_DECREF(list);
    return result;
}

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
        !find(found.step, "tfno_gated_delta_rule_step") || !find(found.recurrence, "tfno_gated_recurrence") ||
        !find(found.recurrence_backward, "tfno_gated_recurrence_backward") || !find(found.recurrence_step, "tfno_gated_recurrence_step") ||
        !find(found.block_norm, "tfno_block_norm") || !find(found.block_norm_backward, "tfno_block_norm_backward") || !find(found.clip, "tfno_clip_grad_norm"))
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
    {"tfno_gated_recurrence", fast(recurrence), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_gated_recurrence_backward", fast(recurrence_backward), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_gated_recurrence_step", fast(recurrence_step), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_block_norm", fast(block_norm), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_block_norm_backward", fast(block_norm_backward), METH_FASTCALL, "The entry point; tensors or addresses for its pointers."},
    {"tfno_clip_grad_norm", fast(clip), METH_FASTCALL, "The entry point for tensors, a limit, the norm's tensor or None, a device and a stream."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
