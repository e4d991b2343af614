// CPython module: the argument marshalling of the entry points around a compressed cache, which a program calls once a layer and token (binding.py).
// A function here takes what its C entry takes, in its order: tensors, addresses or None for pointers, numbers, and a stream (None: torch's current one) at
// the end.  The C declarations say which is which.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

#include "curdkv.h"

namespace {

PyObject *slow_address, *slow_stream, *name_data_ptr;
decltype(&curdkv_rotate) rotate_entry;
decltype(&curdkv_attend) attend_entry;
decltype(&curdkv_compact_mx) compact_mx_entry;
decltype(&curdkv_expand_mx) expand_mx_entry;
decltype(&curdkv_attend_kept) attend_kept_entry;
decltype(&curdkv_attend_kept_mx) attend_kept_mx_entry;
decltype(&curdkv_rotate_axes) rotate_axes_entry;
decltype(&curdkv_attend_weights) attend_weights_entry;
decltype(&curdkv_evict) evict_entry;
decltype(&curdkv_attend_shared) attend_shared_entry;
decltype(&curdkv_attend_shared_mx) attend_shared_mx_entry;

// int(x) as a 64-bit value, wrapped as ctypes wraps it; `ok` false: an error has been set
int64_t integer(PyObject* x, bool& ok) {
    if (!ok) return 0;
    PyObject* made = PyLong_CheckExact(x) ? nullptr : PyNumber_Long(x);
    if (!made && !PyLong_CheckExact(x)) {
        ok = false;
        return 0;
    }
    const unsigned long long r = PyLong_AsUnsignedLongLongMask(made ? made : x);
    if (r == (unsigned long long)-1 && PyErr_Occurred()) ok = false;
    Py_XDECREF(made);
    return (int64_t)r;
}

double real(PyObject* x, bool& ok) {
    if (!ok) return 0.0;
    const double r = PyFloat_AsDouble(x);
    if (r == -1.0 && PyErr_Occurred()) ok = false;
    return r;
}

void* taken(PyObject* x, bool& ok) {
    if (!x) {
        ok = false;
        return nullptr;
    }
    void* r = reinterpret_cast<void*>(integer(x, ok));
    Py_DECREF(x);
    return r;
}

// a tensor's data_ptr(), an integer as it is, None as NULL; anything else is left to Python
void* address(PyObject* x, bool& ok) {
    if (!ok || x == Py_None) return nullptr;
    if (PyLong_CheckExact(x)) return reinterpret_cast<void*>(integer(x, ok));
    PyObject* p = PyObject_CallMethodNoArgs(x, name_data_ptr);
    if (!p && PyErr_ExceptionMatches(PyExc_AttributeError)) {
        PyErr_Clear();
        p = PyObject_CallOneArg(slow_address, x);
    }
    return taken(p, ok);
}

// one argument of the C type T; the last one is the stream
template <class T, bool STREAM>
T argument(PyObject* x, bool& ok) {
    if constexpr (STREAM) {
        if (!ok) return nullptr;
        return PyLong_CheckExact(x) ? reinterpret_cast<void*>(integer(x, ok)) : taken(PyObject_CallOneArg(slow_stream, x), ok);
    } else if constexpr (std::is_pointer_v<T>) return static_cast<T>(address(x, ok));
    else if constexpr (std::is_floating_point_v<T>) return static_cast<T>(real(x, ok));
    else return static_cast<T>(integer(x, ok));
}

template <class... P, size_t... I>
PyObject* called(int (*entry)(P...), PyObject* const* v, Py_ssize_t n, std::index_sequence<I...>) {
    constexpr size_t count = sizeof...(P);
    if (n != (Py_ssize_t)count) {
        PyErr_Format(PyExc_TypeError, "expected %zu arguments, got %zd", count, n);
        return nullptr;
    }
    bool ok = true;
    const std::tuple<P...> args{argument<P, I + 1 == count>(v[I], ok)...};        // (braces: in order)
    if (!ok) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(std::get<I>(args)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
template <class... P>
PyObject* called(int (*entry)(P...), PyObject* const* v, Py_ssize_t n) {
    return called(entry, v, n, std::index_sequence_for<P...>{});
}

#define FUNCTION(f) \
    PyObject* f(PyObject*, PyObject* const* v, Py_ssize_t n) { return called(f##_entry, v, n); }
FUNCTION(rotate)
FUNCTION(attend)
FUNCTION(compact_mx)
FUNCTION(expand_mx)
FUNCTION(attend_kept)
FUNCTION(attend_kept_mx)
FUNCTION(rotate_axes)
FUNCTION(attend_weights)
FUNCTION(evict)
FUNCTION(attend_shared)
FUNCTION(attend_shared_mx)

// bind(addresses of the eleven entries in the order above, address(object) -> int, stream(object) -> int)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 13) {
        PyErr_Format(PyExc_TypeError, "expected 13 arguments, got %zd", n);
        return nullptr;
    }
    bool ok = true;
    void* p[11];
    for (int i = 0; i < 11; ++i) p[i] = reinterpret_cast<void*>(integer(v[i], ok));
    if (!ok) return nullptr;
    rotate_entry = reinterpret_cast<decltype(rotate_entry)>(p[0]);
    attend_entry = reinterpret_cast<decltype(attend_entry)>(p[1]);
    compact_mx_entry = reinterpret_cast<decltype(compact_mx_entry)>(p[2]);
    expand_mx_entry = reinterpret_cast<decltype(expand_mx_entry)>(p[3]);
    attend_kept_entry = reinterpret_cast<decltype(attend_kept_entry)>(p[4]);
    attend_kept_mx_entry = reinterpret_cast<decltype(attend_kept_mx_entry)>(p[5]);
    rotate_axes_entry = reinterpret_cast<decltype(rotate_axes_entry)>(p[6]);
    attend_weights_entry = reinterpret_cast<decltype(attend_weights_entry)>(p[7]);
    evict_entry = reinterpret_cast<decltype(evict_entry)>(p[8]);
    attend_shared_entry = reinterpret_cast<decltype(attend_shared_entry)>(p[9]);
    attend_shared_mx_entry = reinterpret_cast<decltype(attend_shared_mx_entry)>(p[10]);
    Py_INCREF(v[11]);
    Py_XSETREF(slow_address, v[11]);
    Py_INCREF(v[12]);
    Py_XSETREF(slow_stream, v[12]);
    Py_RETURN_NONE;
}

#define ENTRY(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind), ENTRY(rotate), ENTRY(attend), ENTRY(compact_mx), ENTRY(expand_mx), ENTRY(attend_kept), ENTRY(attend_kept_mx),
                         ENTRY(rotate_axes), ENTRY(attend_weights), ENTRY(evict), ENTRY(attend_shared), ENTRY(attend_shared_mx),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attend", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attend(void) {
    name_data_ptr = PyUnicode_InternFromString("data_ptr");
    return name_data_ptr ? PyModule_Create(&module) : nullptr;
}
