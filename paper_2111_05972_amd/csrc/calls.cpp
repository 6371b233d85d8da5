// Python module _calls: the entry points of tp_layer.h whose arguments are numbers and pointers, called without ctypes.  A call of 14 to 22 arguments takes
// about 1 us here and 4 to 5 there (argument by argument, and a method call of Python's for each pointer), against 3 to 5 us of the shortest kernels.
//
// open(path) looks the entry points up in the library at `path`; the functions have their names and take their arguments by place.  A pointer is None, an address, or
// anything with data_ptr() (a tensor) or cuda_stream (a stream), what int() takes or a ctypes pointer; numbers may be ctypes' too.  Numbers that do not fit their argument raise OverflowError.  Other threads run during a call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>

#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/tp_layer.h"

#define ENTRY_POINTS(X)                                                                                                        \
    X(ln_workspace_bytes) X(ln_fwd) X(ln_bwd) X(ln_moments) X(ln_stats) X(ln_apply_fwd) X(ln_apply_bwd_sums)                   \
    X(ln_apply_workspace_bytes) X(ln_apply_bwd) X(slice_epilogue_fwd) X(slice_epilogue_workspace_bytes) X(slice_epilogue_bwd)  \
    X(dropout_fwd) X(dropout_workspace_bytes) X(dropout_bwd) X(slice_epilogue_bwd_static)                                      \
    X(gemm_workspace_bytes) X(gemm) X(attn_workspace_bytes) X(attn_fwd) X(attn_bwd) X(rope_fwd) X(rope_bwd)                    \
    X(qk_norm_rope_fwd) X(qk_norm_rope_workspace_bytes) X(qk_norm_rope_bwd) X(pack_plan_bytes) X(pack_plan)                    \
    X(attn_packed_workspace_bytes) X(attn_packed_fwd) X(attn_packed_bwd) X(window_plan_bytes) X(window_plan)                   \
    X(attn_window_workspace_bytes) X(attn_window_fwd) X(attn_window_bwd) X(lm_loss_workspace_bytes) X(lm_loss_fwd)             \
    X(lm_loss_join) X(lm_loss_bwd)

namespace {

#define X(name) I_##name,
enum Index { ENTRY_POINTS(X) COUNT };
#undef X
void* table[COUNT];
PyObject *data_ptr_name, *cuda_stream_name;
PyTypeObject* stream_type;      // of the last object that had no data_ptr(): asked for its stream at once
PyObject* ctypes_value;         // the class of ctypes' numbers and pointers

// The value of one of those (a new reference), or null without an error.
PyObject* value_of(PyObject* o) {
    const int is = PyObject_IsInstance(o, ctypes_value);
    if (is <= 0) { PyErr_Clear(); return nullptr; }
    PyObject* value = PyObject_GetAttrString(o, "value");
    if (!value) PyErr_Clear();
    return value;
}
// What int() takes (numpy's integers), or the value of a ctypes pointer, None included.
PyObject* other_number(PyObject* o) {
    PyObject* number = PyNumber_Long(o);
    if (number) return number;
    PyErr_Clear();
    PyObject* value = value_of(o);
    if (value) {
        number = value == Py_None ? PyLong_FromLong(0) : PyNumber_Index(value);
        Py_DECREF(value);
    }
    if (!number) PyErr_Format(PyExc_TypeError, "a pointer is None, an address, a tensor or a stream, not %s", Py_TYPE(o)->tp_name);
    return number;
}
// Null without an error: it has no such attribute.
PyObject* data_ptr_of(PyObject* o) {
    PyObject* self[2] = {nullptr, o};
    PyObject* number = PyObject_VectorcallMethod(data_ptr_name, self + 1, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
    if (!number && PyErr_ExceptionMatches(PyExc_AttributeError)) PyErr_Clear();
    return number;
}
PyObject* stream_of(PyObject* o) {
    PyObject* number = PyObject_GetAttr(o, cuda_stream_name);
    if (number && Py_TYPE(o) != stream_type) {
        Py_INCREF(Py_TYPE(o));
        Py_XSETREF(stream_type, Py_TYPE(o));
    } else if (!number && PyErr_ExceptionMatches(PyExc_AttributeError)) {
        PyErr_Clear();
    }
    return number;
}
bool address(PyObject* o, void** out) {
    if (o == Py_None) { *out = nullptr; return true; }
    PyObject* number = nullptr;
    if (PyLong_Check(o)) {
        number = Py_NewRef(o);
    } else {
        const bool stream = Py_TYPE(o) == stream_type;
        number = stream ? stream_of(o) : data_ptr_of(o);
        if (!number && !PyErr_Occurred()) number = stream ? data_ptr_of(o) : stream_of(o);
        if (!number && !PyErr_Occurred()) number = other_number(o);
        if (!number) return false;
    }
    *out = PyLong_AsVoidPtr(number);
    Py_DECREF(number);
    return !(*out == nullptr && PyErr_Occurred());
}
template <typename T> bool convert(PyObject* o, T* out);
// A number that ctypes made, after the error that it is none.
template <typename T> bool of_ctypes(PyObject* o, T* out) {
    if (!PyErr_ExceptionMatches(PyExc_TypeError)) return false;
    PyObject *type, *error, *trace;
    PyErr_Fetch(&type, &error, &trace);
    PyObject* value = value_of(o);
    if (!value) { PyErr_Restore(type, error, trace); return false; }
    Py_XDECREF(type);
    Py_XDECREF(error);
    Py_XDECREF(trace);
    const bool ok = convert(value, out);
    Py_DECREF(value);
    return ok;
}
template <typename T> bool convert(PyObject* o, T* out) {
    if constexpr (std::is_pointer_v<T>) {
        void* p;
        if (!address(o, &p)) return false;
        *out = static_cast<T>(p);
        return true;
    } else if constexpr (std::is_floating_point_v<T>) {
        const double v = PyFloat_AsDouble(o);
        *out = (T)v;
        return !(v == -1.0 && PyErr_Occurred()) || of_ctypes(o, out);
    } else {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) return of_ctypes(o, out);
        const bool fits = std::is_signed_v<T> ? v >= (long long)std::numeric_limits<T>::min() && v <= (long long)std::numeric_limits<T>::max() : v >= 0;
        if (!fits) { PyErr_SetString(PyExc_OverflowError, "a number does not fit its argument"); return false; }
        *out = (T)v;
        return true;
    }
}

template <int I, typename Sig> struct Entry;
template <int I, typename R, typename... A> struct Entry<I, R(A...)> {
    template <size_t... N>
    static PyObject* call(PyObject* const* args, std::index_sequence<N...>) {
        std::tuple<A...> a{};
        if (!(convert(args[N], &std::get<N>(a)) && ...)) return nullptr;
        if (!table[I]) { PyErr_SetString(PyExc_RuntimeError, "open() comes first"); return nullptr; }
        const auto f = reinterpret_cast<R (*)(A...)>(table[I]);
        R r;
        Py_BEGIN_ALLOW_THREADS
        r = f(std::get<N>(a)...);
        Py_END_ALLOW_THREADS
        if constexpr (std::is_same_v<R, size_t>) return PyLong_FromSize_t(r);
        else return PyLong_FromLong(r);
    }
    static PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
        if (n != (Py_ssize_t)sizeof...(A)) {
            PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, (Py_ssize_t)sizeof...(A));
            return nullptr;
        }
        return call(args, std::index_sequence_for<A...>{});
    }
};

PyObject* open_library(PyObject*, PyObject* path) {
    const char* p = PyUnicode_AsUTF8(path);
    if (!p) return nullptr;
    void* lib = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    if (!lib) { PyErr_SetString(PyExc_ImportError, dlerror()); return nullptr; }
#define X(name) "tp_layer_" #name,
    const char* const names[COUNT] = {ENTRY_POINTS(X)};
#undef X
    for (int i = 0; i < COUNT; ++i)
        if (!(table[i] = dlsym(lib, names[i]))) { PyErr_Format(PyExc_ImportError, "%s: no %s", p, names[i]); return nullptr; }
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
#define X(name) {"tp_layer_" #name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&Entry<I_##name, decltype(tp_layer_##name)>::entry)), METH_FASTCALL, nullptr},
    ENTRY_POINTS(X)
#undef X
    {"open", open_library, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    PyObject* ctypes = PyImport_ImportModule("_ctypes");
    if (!ctypes) return nullptr;
    ctypes_value = PyObject_GetAttrString(ctypes, "_SimpleCData");
    Py_DECREF(ctypes);
    if (!ctypes_value) return nullptr;
    data_ptr_name = PyUnicode_InternFromString("data_ptr");
    cuda_stream_name = PyUnicode_InternFromString("cuda_stream");
    return data_ptr_name && cuda_stream_name ? PyModule_Create(&module) : nullptr;
}
